"""CPU-side tests of the operators of a training step around a routed layer: pins of their oracle, gradients against differences, and
the argument checks of the entry points, all of which refuse before any CUDA call."""
import ctypes

import numpy as np
import pytest
import torch

import oracle

FAKE = 0x10000      # an aligned address that is never dereferenced: the checks below fail first


# ----------------------------------------------------------------------------- oracle pins

def test_sorted_order_pins():
    select = np.array([[1, 0, 1], [0, 0, 0], [1, 1, 1], [0, 0, 7]], np.uint8)
    r = oracle.sort_tokens(select, 2, 1)
    assert r["counts"].tolist() == [2, 1, 2] and r["offsets"].tolist() == [0, 2, 3, 5]          # token 2's third branch is past its slots
    assert r["row_token"].tolist() == [0, 2, 2, 0, 3]
    assert r["token_row"].tolist() == [[0, 3], [-1, -1], [1, 2], [4, -1]] and r["token_branch"].tolist() == [[0, 2], [-1, -1], [0, 1], [2, -1]]
    r = oracle.sort_tokens(select, 2, 4)
    assert r["offsets"].tolist() == [0, 4, 8, 12] and r["row_token"].tolist() == [0, 2, -1, -1, 2, -1, -1, -1, 0, 3, -1, -1]


@pytest.mark.parametrize("n,B,slots,align", [(50, 7, 3, 1), (33, 20, 20, 8), (1, 1, 1, 16)])
def test_sorted_order_is_an_order(n, B, slots, align):
    rng = np.random.default_rng(n)
    select = (rng.uniform(size=(n, B)) < 0.3).astype(np.uint8)
    r = oracle.sort_tokens(select, slots, align)
    for b in range(B):
        own = r["row_token"][r["offsets"][b]:r["offsets"][b] + r["counts"][b]]
        assert np.all(np.diff(own) > 0) and all(select[t, b] for t in own) and r["offsets"][b] % align == 0
    assert r["counts"].sum() == sum(min(int(s.sum()), slots) for s in select)
    x = rng.normal(size=(n, 3))
    rows = np.where(r["row_token"][:, None] >= 0, x[r["row_token"]], 0.0)
    # there and back without weights: every token as often as it has branches
    back = oracle.combine(rows, r["token_row"])
    assert np.allclose(back, x * (r["token_row"] >= 0).sum(axis=1, keepdims=True))


def test_combine_gradient_is_the_differences():
    rng = np.random.default_rng(1)
    select = (rng.uniform(size=(6, 4)) < 0.6).astype(np.uint8)
    plan = oracle.sort_tokens(select, 3, 2)
    rows, w, gy = rng.normal(size=(len(plan["row_token"]), 5)), rng.normal(size=(6, 3)), rng.normal(size=(6, 5))
    grad_rows, grad_w = oracle.combine_grad(gy, rows, plan["token_row"], w)

    def loss(rows, w):
        return float((oracle.combine(rows, plan["token_row"], w, np.ones((6, 5))) * gy).sum())
    for at in np.ndindex(rows.shape):
        up, dn = rows.copy(), rows.copy()
        up[at] += 1e-5
        dn[at] -= 1e-5
        assert abs((loss(up, w) - loss(dn, w)) / 2e-5 - grad_rows[at]) < 1e-8
    for at in np.ndindex(w.shape):
        up, dn = w.copy(), w.copy()
        up[at] += 1e-5
        dn[at] -= 1e-5
        assert abs((loss(rows, up) - loss(rows, dn)) / 2e-5 - grad_w[at]) < 1e-8


@pytest.mark.parametrize("layer", [False, True])
def test_norm_gradient_is_the_differences(layer):
    rng = np.random.default_rng(2)
    s, gain, bias, gv, gs = rng.normal(size=(3, 6)) + 0.5, rng.normal(size=6), rng.normal(size=6), rng.normal(size=(3, 6)), rng.normal(size=(3, 6))

    def loss(s, gain, bias):
        out = oracle.add_layernorm(s, None, gain, bias, 1e-3)[1] if layer else oracle.add_rmsnorm(s, None, gain, 1e-3)[1]
        return float((out * gv).sum() + (s * gs).sum())
    dx, dg, db = oracle.norm_grad(layer, s, gain, gv, gs, 1e-3)
    for value, grad in ((s, dx), (gain, dg)) + (((bias, db),) if layer else ()):
        for at in np.ndindex(value.shape):
            keep = value[at]
            value[at] = keep + 1e-5
            up = loss(s, gain, bias)
            value[at] = keep - 1e-5
            down = loss(s, gain, bias)
            value[at] = keep
            assert abs((up - down) / 2e-5 - grad[at]) < 1e-7


def test_layernorm_against_torch():
    rng = np.random.default_rng(3)
    x, r, gain, bias = rng.normal(size=(4, 9)), rng.normal(size=(4, 9)), rng.normal(size=9), rng.normal(size=9)
    want = torch.nn.functional.layer_norm(torch.from_numpy(x + r), (9,), torch.from_numpy(gain), torch.from_numpy(bias), 1e-4).numpy()
    assert np.allclose(oracle.add_layernorm(x, r, gain, bias, 1e-4)[1], want, rtol=1e-12)


def test_adamw_against_torch():
    rng = np.random.default_rng(4)
    p = torch.from_numpy(rng.normal(size=17)).requires_grad_()
    opt = torch.optim.AdamW([p], lr=3e-2, betas=(0.8, 0.95), eps=1e-6, weight_decay=0.2)
    q, m, v = p.detach().numpy().copy(), np.zeros(17), np.zeros(17)
    for step in range(1, 6):
        g = rng.normal(size=17)
        p.grad = torch.from_numpy(g.copy())
        opt.step()
        q, m, v = oracle.adamw(q, g, m, v, 3e-2, 0.8, 0.95, 1e-6, 0.2, step)
        assert np.allclose(q, p.detach().numpy(), rtol=1e-12, atol=1e-14)


def test_adamw_noise_pins():
    assert oracle.mix32(0) == 0 and oracle.mix32(1) == 0x514E28B7      # MurmurHash3's own
    seed, step, tensor = 0x123456789ABCDEF, 7, 3
    noise = oracle.adamw_noise(seed, step, tensor, 300000)
    key = oracle.mix32(tensor ^ oracle.mix32(oracle.mix32(oracle.mix32(seed & 0xFFFFFFFF) ^ (seed >> 32)) ^ step))
    assert [int(noise[i]) for i in (0, 1, 99999)] == [oracle.mix32((key + i * 0x9E3779B1) & 0xFFFFFFFF) for i in (0, 1, 99999)]
    # each half is uniform: mean 1/2 within five deviations of 1 / sqrt(12 n), and the halves are not correlated
    a, b = (noise & np.uint64(0xFFFF)).astype(float) / 65536, (noise >> np.uint64(16)).astype(float) / 65536
    assert max(abs(a.mean() - 0.5), abs(b.mean() - 0.5)) < 5 / np.sqrt(12 * 300000) and abs(np.corrcoef(a, b)[0, 1]) < 5 / np.sqrt(300000)
    other = oracle.adamw_noise(seed, step + 1, tensor, 300000)
    assert abs(np.corrcoef(noise.astype(float), other.astype(float))[0, 1]) < 5 / np.sqrt(300000)


def test_stochastic_codes_have_the_right_mean():
    rng = np.random.default_rng(5)
    for a in (0.001, 2.0 ** -7, 0.3, 1.01, 5.5, 300.0, 447.9):
        codes = oracle.e4m3_up_or_down(np.full(200000, a), rng.integers(0, 65536, 200000))
        step = 2.0 ** (np.floor(np.log2(max(a, 2.0 ** -6))) - 3)
        assert set(np.unique(codes)) <= {np.floor(a / step) * step, (np.floor(a / step) + 1) * step}
        # a coin of deviation step / 2 at most, 200000 times
        assert abs(codes.mean() - a) < 5 * step / 2 / np.sqrt(200000) + step * 2.0 ** -17
    assert oracle.e4m3_up_or_down(np.array([448.0, 0.0]), np.array([65535, 65535])).tolist() == [448.0, 0.0]


def test_roots_above_zero_stay_above_zero():
    x = np.zeros(130)
    x[:3] = 1.0, 1e-9, 1e-30
    codes, scales = oracle.adamw_blocks(x, True)
    assert codes[:4].tolist() == [448.0, 2.0 ** -9, 2.0 ** -9, 0.0] and scales[1] == 2.0 ** -126
    codes, _ = oracle.adamw_blocks(x, True, np.zeros(130, np.uint64))
    assert codes[:4].tolist() == [448.0, 2.0 ** -9, 2.0 ** -9, 0.0]


# ----------------------------------------------------------------------------- sizes and refusals

def test_sort_sizes(lib):
    assert lib.mlpmoe_sort_rows(0, 8, 2) == 0 and lib.mlpmoe_sort_rows(10, 8, 2) == 20
    assert lib.mlpmoe_sort_rows(10, 3, 5, 16) == 30 + 3 * 15           # a token has no more branches than there are
    assert lib.mlpmoe_sort_rows(1, 64, 2, 128) == 2 + 2 * 127          # nor do more branches have rows than there are rows
    for n in (0, 1, 1024, 1025, 40000, 700000):
        for B in (1, 32, 33, 256):
            assert lib.mlpmoe_sort_workspace(n, B) >= 16
    for B in (3, 40, 64, 128, 250):                                     # a workspace serves every smaller batch
        sizes = [lib.mlpmoe_sort_workspace(n, B) for n in range(0, 120000, 31)] + [lib.mlpmoe_sort_workspace(n, B) for n in range(10 ** 6, 10 ** 7, 99991)]
        assert sizes == sorted(sizes)
    for call in (lambda: lib.mlpmoe_sort_rows(-1, 8, 2), lambda: lib.mlpmoe_sort_rows(1, 0, 2), lambda: lib.mlpmoe_sort_rows(1, 8, 0),
                 lambda: lib.mlpmoe_sort_rows(1, 8, 2, 0), lambda: lib.mlpmoe_sort_workspace(-1, 8), lambda: lib.mlpmoe_sort_workspace(1, 0)):
        with pytest.raises(lib.MlpmoeError) as e:
            call()
        assert e.value.status == lib.MLPMOE_ERR_INVALID_ARG
    for call in (lambda: lib.mlpmoe_sort_rows(1, 257, 2), lambda: lib.mlpmoe_sort_rows(1, 8, 2, 1025), lambda: lib.mlpmoe_sort_workspace(1, 257),
                 lambda: lib.mlpmoe_sort_rows(2 ** 30, 8, 2), lambda: lib.mlpmoe_sort_rows(2 ** 31 - 1, 8, 1, 2)):
        with pytest.raises(lib.MlpmoeError) as e:
            call()
        assert e.value.status == lib.MLPMOE_ERR_UNSUPPORTED


def test_sort_refusals(lib):
    ws = lib.mlpmoe_sort_workspace(100, 8)

    def call(sel=FAKE, n=100, B=8, slots=2, align=1, off=FAKE, cnt=FAKE, rt=FAKE, rows=200, tr=FAKE, tb=None, w=FAKE, wb=ws):
        return lib.lib.mlpmoe_sort_tokens(sel, n, B, slots, align, off, cnt, rt, rows, tr, tb, w, wb, None)

    for kw in (dict(sel=None), dict(n=-1), dict(B=0), dict(slots=0), dict(align=0), dict(off=None), dict(cnt=None), dict(rt=None), dict(rows=199),
               dict(align=4, rows=200 + 23), dict(rows=2 ** 31), dict(tr=None), dict(w=None), dict(wb=ws - 1), dict(w=FAKE + 8), dict(off=FAKE + 2),
               dict(cnt=FAKE + 1), dict(rt=FAKE + 2), dict(tr=FAKE + 2), dict(tb=FAKE + 1)):
        assert call(**kw) == lib.MLPMOE_ERR_INVALID_ARG, kw
    for kw in (dict(B=257), dict(align=1025), dict(n=2 ** 31 - 1)):
        assert call(**kw) == lib.MLPMOE_ERR_UNSUPPORTED, kw


def test_dispatch_refusals(lib):
    def call(x=FAKE, t=0, xs=0, sc=FAKE, g=0, n=10, d=64, B=8, slots=2, align=1, off=FAKE, cnt=FAKE, tr=FAKE, rows=FAKE, rs=0, rsc=FAKE, nr=20):
        return lib.lib.mlpmoe_dispatch(x, t, xs, sc, g, n, d, B, slots, align, off, cnt, tr, rows, rs, rsc, nr, None)

    assert call(n=0, x=None, rows=None, tr=None) == lib.MLPMOE_OK
    for kw in (dict(x=None), dict(t=3), dict(xs=63), dict(rs=63), dict(n=-1), dict(d=0), dict(B=0), dict(slots=0), dict(align=0), dict(tr=None),
               dict(rows=None), dict(nr=-1), dict(nr=2 ** 31), dict(t=2, g=48), dict(t=2, sc=None), dict(t=2, rsc=None), dict(t=2, sc=FAKE + 2),
               dict(t=2, rsc=FAKE + 1), dict(x=FAKE + 1), dict(rows=FAKE + 1), dict(t=1, x=FAKE + 2), dict(tr=FAKE + 2), dict(align=2, off=None),
               dict(align=2, cnt=None), dict(align=2, off=FAKE + 2), dict(align=2, cnt=FAKE + 1)):
        assert call(**kw) == lib.MLPMOE_ERR_INVALID_ARG, kw
    for kw in (dict(B=257), dict(align=1025), dict(n=2 ** 31 - 1, d=65536, nr=2 ** 31 - 1)):
        assert call(**kw) == lib.MLPMOE_ERR_UNSUPPORTED, kw


def test_combine_refusals(lib):
    def call(rows=FAKE, rt=0, rs=0, nr=20, tr=FAKE, w=FAKE, slots=2, res=None, rest=1, ress=0, y=FAKE + 4096, yt=1, ys=0, n=10, d=64):
        return lib.lib.mlpmoe_combine(rows, rt, rs, nr, tr, w, slots, res, rest, ress, y, yt, ys, n, d, None)

    assert call(n=0, rows=None, tr=None, y=None) == lib.MLPMOE_OK
    for kw in (dict(rows=None), dict(rt=2), dict(yt=2), dict(res=FAKE, rest=2), dict(rs=63), dict(ys=63), dict(res=FAKE, ress=63), dict(nr=-1),
               dict(nr=2 ** 31), dict(tr=None), dict(slots=0), dict(y=None), dict(n=-1), dict(d=0), dict(rows=FAKE + 1), dict(tr=FAKE + 2),
               dict(w=FAKE + 2), dict(y=FAKE + 2), dict(res=FAKE + 2), dict(res=FAKE + 4096, rest=0), dict(res=FAKE + 4096, ress=72)):
        assert call(**kw) == lib.MLPMOE_ERR_INVALID_ARG, kw
    assert call(n=2 ** 31 - 1, d=65536) == lib.MLPMOE_ERR_UNSUPPORTED


def test_combine_backward_refusals(lib):
    def call(gy=FAKE, gt=1, gs=0, rows=FAKE, rt=0, rs=0, nr=20, tr=FAKE, w=FAKE, slots=2, B=8, align=1, off=FAKE, cnt=FAKE, gr=FAKE + 4096, grs=0,
             gw=FAKE, n=10, d=64):
        return lib.lib.mlpmoe_combine_backward(gy, gt, gs, rows, rt, rs, nr, tr, w, slots, B, align, off, cnt, gr, grs, gw, n, d, None)

    assert call(n=0, gy=None, tr=None) == lib.MLPMOE_OK
    for kw in (dict(gy=None), dict(gt=2), dict(rt=2), dict(gs=63), dict(rs=63), dict(grs=63), dict(rows=None), dict(nr=-1), dict(tr=None), dict(slots=0),
               dict(B=0), dict(align=0), dict(gr=None, gw=None), dict(n=-1), dict(d=0), dict(gy=FAKE + 2), dict(rows=FAKE + 1), dict(gr=FAKE + 1),
               dict(gw=FAKE + 2), dict(w=FAKE + 1), dict(tr=FAKE + 1), dict(align=2, off=None), dict(align=2, cnt=None), dict(align=2, off=FAKE + 1),
               dict(gr=FAKE, rs=64, grs=72)):
        assert call(**kw) == lib.MLPMOE_ERR_INVALID_ARG, kw
    for kw in (dict(d=32769), dict(B=257), dict(align=1025), dict(n=2 ** 31 - 1)):
        assert call(**kw) == lib.MLPMOE_ERR_UNSUPPORTED, kw


def test_add_layernorm_refusals(lib):
    f = lib.lib.mlpmoe_add_layernorm

    def call(x=FAKE, xt=1, xs=0, r=FAKE, rt=0, rs=0, gain=FAKE, bias=FAKE, xo=FAKE, xos=0, out=FAKE, ot=0, os_=0, scales=FAKE, group=0, n=4, d=64):
        return f(x, xt, xs, r, rt, rs, gain, bias, xo, xos, out, ot, os_, scales, group, n, d, 1e-5, None)

    assert call(n=0) == lib.MLPMOE_OK
    for kw in (dict(n=-1), dict(d=0), dict(x=None), dict(out=None), dict(xt=2), dict(rt=2), dict(ot=3), dict(ot=2, scales=None), dict(ot=2, group=48),
               dict(xs=63), dict(rs=63), dict(xos=63), dict(os_=63), dict(x=FAKE + 2), dict(gain=FAKE + 2), dict(bias=FAKE + 2), dict(out=FAKE + 1)):
        assert call(**kw) == lib.MLPMOE_ERR_INVALID_ARG, kw
    assert call(d=32769) == lib.MLPMOE_ERR_UNSUPPORTED


def test_norm_backward_refusals(lib):
    size = lib.mlpmoe_norm_backward_workspace(10, 64)
    assert lib.mlpmoe_norm_backward_workspace(0, 64) > 0
    for d in (8, 256, 257, 1024, 2000, 4096, 8192, 8193, 32768):        # a workspace serves every smaller batch
        sizes = [lib.mlpmoe_norm_backward_workspace(n, d) for n in range(0, 20000, 7)]
        assert sizes == sorted(sizes)

    def call(k=1, s=FAKE, st=1, ss=0, gain=FAKE, go=FAKE, got=0, gos=0, gs=None, gst=1, gss=0, gx=FAKE + 4096, gxt=1, gxs=0, gg=FAKE, gb=FAKE, n=10, d=64,
             w=FAKE, wb=size):
        return lib.lib.mlpmoe_norm_backward(k, s, st, ss, gain, go, got, gos, gs, gst, gss, gx, gxt, gxs, gg, gb, n, d, 1e-5, w, wb, None)

    assert call(n=0, gg=None, gb=None, w=None) == lib.MLPMOE_OK
    for kw in (dict(k=2), dict(k=0), dict(s=None), dict(st=2), dict(ss=63), dict(go=None), dict(got=2), dict(gos=63), dict(gs=FAKE, gst=2),
               dict(gs=FAKE, gss=63), dict(gx=None), dict(gxt=2), dict(gxs=63), dict(gx=FAKE), dict(gs=FAKE + 4096, gst=0),
               dict(gs=FAKE + 4096, gss=72), dict(n=-1), dict(d=0), dict(w=None), dict(wb=size - 1), dict(w=FAKE + 8), dict(s=FAKE + 2), dict(gain=FAKE + 2),
               dict(go=FAKE + 1), dict(gs=FAKE + 2), dict(gx=FAKE + 2), dict(gg=FAKE + 2), dict(gb=FAKE + 2)):
        assert call(**kw) == lib.MLPMOE_ERR_INVALID_ARG, kw      # k = 0: RMSNorm has no bias
    assert call(d=32769) == lib.MLPMOE_ERR_UNSUPPORTED
    with pytest.raises(lib.MlpmoeError):
        lib.mlpmoe_norm_backward_workspace(1, 32769)


def test_adamw_refusals(lib):
    def call(step=1, lr=1e-3, b1=0.9, b2=0.999, eps=1e-8, step_device=None, lr_device=None, scale=None, count=1, settings=True, **t):
        record = dict(n=10, param=FAKE, grad=FAKE, m=FAKE, v=FAKE) | t
        arr = lib.mlpmoe_adamw_tensors([record])
        o = lib.mlpmoe_adamw_settings_t(lr, b1, b2, eps, step, step_device, lr_device, scale, 0, 0)
        return lib.lib.mlpmoe_adamw(arr if count else None, count, ctypes.byref(o) if settings else None, None)

    nan = float("nan")
    assert call(count=0) == lib.MLPMOE_OK and call(n=0, param=None) == lib.MLPMOE_OK
    for kw in (dict(count=-1), dict(settings=False), dict(step=0), dict(b1=1.0), dict(b1=-0.1), dict(b2=1.0), dict(b2=nan), dict(eps=0.0), dict(eps=1e-60),
               dict(eps=nan), dict(lr=nan), dict(lr=float("inf")), dict(step_device=FAKE + 4), dict(lr_device=FAKE + 2), dict(scale=FAKE + 2), dict(n=-1),
               dict(weight_decay=-1.0), dict(weight_decay=nan), dict(param=None), dict(grad=None), dict(m=None), dict(v=None), dict(param_dtype=2),
               dict(grad_dtype=2), dict(state_dtype=0), dict(state_dtype=2), dict(state_dtype=2, m_scale=FAKE, v_scale=FAKE + 2),
               dict(param_dtype=0, param_bf16=FAKE), dict(param_bf16=FAKE + 1), dict(param=FAKE + 2), dict(grad=FAKE + 2), dict(m=FAKE + 1),
               dict(v=FAKE + 2)):
        assert call(**kw) == lib.MLPMOE_ERR_INVALID_ARG, kw
    assert lib.lib.mlpmoe_adamw(None, 1, ctypes.byref(lib.mlpmoe_adamw_settings_t(1e-3, 0.9, 0.999, 1e-8, 1)), None) == lib.MLPMOE_ERR_INVALID_ARG
    assert call(n=2 ** 40 + 1) == lib.MLPMOE_ERR_UNSUPPORTED
