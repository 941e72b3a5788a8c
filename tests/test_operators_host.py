"""CPU-side tests of the operators around a routed layer step: pins of their oracle, and the argument checks of the
entry points, all of which refuse before any CUDA call."""
import ctypes

import numpy as np
import pytest
import torch

import oracle

FAKE = 0x10000      # an aligned address that is never dereferenced: the checks below fail first


# ----------------------------------------------------------------------------- oracle pins

def test_e4m3_rounding_against_torch():
    rng = np.random.default_rng(0)
    a = np.concatenate([rng.normal(size=4000) * 10.0 ** rng.uniform(-4, 2.6, 4000), np.linspace(-500, 500, 3001),
                        np.arange(-64, 65) * 2.0 ** -11, [0.0, 448.0, 464.0, 1e9]]).astype(np.float32)
    a = np.clip(a, -448, 448)
    want = torch.from_numpy(a).to(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(oracle.round_to_e4m3(a), want)


def test_quantize_e4m3_bounds():
    rng = np.random.default_rng(1)
    v = rng.normal(size=(5, 200))
    v[1] = 0.0
    for group in (0, 32, 64, 128):
        codes, scales = oracle.quantize_e4m3(v, group)
        back = codes * np.repeat(scales, group or 200, axis=1)[:, :200]
        # half a step: 2^-4 of the value, or half the smallest step 2^-9 of the scale
        assert np.all(np.abs(back - v) <= np.maximum(np.abs(v) * 2.0 ** -4, 2.0 ** -10 * np.repeat(scales, group or 200, axis=1)[:, :200]) * (1 + 1e-12))
        assert np.all(scales[1] == 2.0 ** -126) and np.all(codes[1] == 0)


def test_route_pins():
    # uniform logits: every probability 1 / B, and with the ties to the lowest index the first k branches take all tokens
    r = oracle.route(np.zeros((7, 5)), 2)
    assert np.array_equal(r["counts"], [7, 7, 0, 0, 0, 7]) and np.allclose(r["prob"], 0.2) and np.isclose(r["loss"], 5 * (0.5 * 0.2 * 2))
    # balanced one-hot-like routing has loss 1 when prob is uniform over the branches
    logits = np.eye(4) * 50
    r = oracle.route(logits, 1)
    assert np.array_equal(r["counts"], [1, 1, 1, 1, 4]) and np.isclose(r["loss"], 1.0)
    # nothing eligible
    r = oracle.route(np.full((3, 4), -np.inf), 2)
    assert r["counts"].sum() == 0 and r["loss"] == 0.0 and np.all(r["prob"] == 0)
    r = oracle.route(np.array([[1.0, np.nan, -np.inf, 0.5]]), 3)
    assert r["select"].tolist() == [[1, 0, 0, 1]]


def test_route_grad_against_differences():
    rng = np.random.default_rng(2)
    logits = rng.normal(size=(6, 5))
    logits[0, 2] = -np.inf
    avail, valid = np.array([1, 1, 1, 1, 0]), np.array([1, 1, 0, 1, 1, 1])
    counts = oracle.route(logits, 2, avail, valid)["counts"]
    grad, _ = oracle.route_grad(logits, counts, avail, valid, 1.7)

    def loss(x):          # the loss at constant counts
        r = oracle.route(x, 2, avail, valid)
        return 1.7 * 4 * float(np.dot(counts[:-1] / counts[:-1].sum(), r["p"].sum(axis=0) / counts[-1]))
    for t in range(6):
        for b in range(5):
            if not np.isfinite(logits[t, b]):
                assert grad[t, b] == 0
                continue
            up, dn = logits.copy(), logits.copy()
            up[t, b] += 1e-5
            dn[t, b] -= 1e-5
            assert abs((loss(up) - loss(dn)) / 2e-5 - grad[t, b]) < 1e-8
    assert np.allclose(grad.sum(axis=1), 0.0)


@pytest.mark.parametrize("asym", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_w4_oracle_round_trip(group, asym):
    rng = np.random.default_rng(3)
    W = (rng.normal(size=(24, 200)) * 0.02).astype(np.float32)
    W[3] = 0.0
    W[5] = np.abs(W[5])
    c, s, z = oracle.w4_quantize(W, group, asym)
    back = oracle.w4_dequantize(c, s, z, group)
    step = np.repeat(s.T, group, axis=1)[:, :200]
    # half a step; the scale's own rounding to bf16 and the zero's rounding cost up to another half at the range's ends
    assert np.all(np.abs(back - W) <= step * (1.0 + 8 * 2.0 ** -8) + 1e-12)
    assert np.all(back[3] == 0)
    q, _, _ = oracle.w4_pack(c, s, z, pad=15)
    assert np.array_equal(oracle.w4_unpack(q, 24, 200), c)


def test_w4_layer_is_the_layer_equation():
    rng = np.random.default_rng(4)
    d, d_b = 16, [16, 32, 16]
    I = sum(d_b)
    Wg, Wu, Wd = rng.normal(size=(I, d)), rng.normal(size=(I, d)), rng.normal(size=(d, I))
    x, alpha = rng.normal(size=(5, d)), [1.0, -0.5, 0.8]
    got = oracle.w4_layer_forward(x, Wg, Wu, Wd, d_b, alpha)["y"]
    assert np.allclose(got, oracle.mlpmoe_forward(x, Wg.T, Wu.T, Wd.T, d_b, alpha), rtol=1e-12)
    sel = (rng.uniform(size=(5, 3)) < 0.5).astype(np.uint8)
    got = oracle.w4_layer_forward(x, Wg, Wu, Wd, d_b, alpha, sel)["y"]
    assert np.allclose(got, oracle.routed_forward(x, Wg.T, Wu.T, Wd.T, d_b, alpha, sel), rtol=1e-12)


# ----------------------------------------------------------------------------- refusals

def test_add_rmsnorm_refusals(lib):
    f = lib.lib.mlpmoe_add_rmsnorm

    def call(x=FAKE, xt=1, xs=0, r=FAKE, rt=0, rs=0, gain=FAKE, xo=FAKE, xos=0, out=FAKE, ot=0, os_=0, scales=FAKE, group=0, n=4, d=64):
        return f(x, xt, xs, r, rt, rs, gain, xo, xos, out, ot, os_, scales, group, n, d, 1e-6, None)

    bad = lib.MLPMOE_ERR_INVALID_ARG
    assert call(n=0) == lib.MLPMOE_OK                                            # nothing to do
    for kw in (dict(n=-1), dict(d=0), dict(x=None), dict(out=None), dict(xt=2), dict(rt=2), dict(ot=3), dict(ot=2, scales=None),
               dict(ot=2, group=48), dict(ot=2, group=-1), dict(xs=63), dict(rs=63), dict(xos=63), dict(os_=63), dict(x=FAKE + 2), dict(r=FAKE + 1),
               dict(gain=FAKE + 2), dict(xo=FAKE + 1), dict(out=FAKE + 1), dict(ot=2, scales=FAKE + 2), dict(xo=FAKE, xs=64, xos=72)):
        assert call(**kw) == bad, kw
    assert call(d=32769) == lib.MLPMOE_ERR_UNSUPPORTED
    # the plain norm writes fp32 or bf16 only
    assert lib.lib.mlpmoe_rmsnorm(FAKE, FAKE, 4, 64, 1e-6, lib.MLPMOE_E4M3, None) == bad


def test_route_refusals(lib):
    size = ctypes.c_int64()
    assert lib.lib.mlpmoe_route_workspace(10, 8, ctypes.byref(size)) == lib.MLPMOE_OK and size.value > 0
    ws = size.value
    bad = lib.MLPMOE_ERR_INVALID_ARG

    def call(x=FAKE, dt=1, st=0, n=10, B=8, k=2, sel=FAKE, cnt=FAKE, prob=FAKE, loss=FAKE, w=FAKE, wb=ws):
        return lib.lib.mlpmoe_route(x, dt, st, n, B, k, None, None, sel, cnt, prob, loss, w, wb, None)

    for kw in (dict(x=None), dict(dt=2), dict(st=7), dict(n=-1), dict(B=0), dict(k=0), dict(k=9), dict(sel=None), dict(cnt=None), dict(prob=None),
               dict(loss=None), dict(w=None), dict(wb=ws - 1), dict(w=FAKE + 4), dict(x=FAKE + 2), dict(cnt=FAKE + 1)):
        assert call(**kw) == bad, kw
    assert call(B=257, k=1) == lib.MLPMOE_ERR_UNSUPPORTED

    def back(x=FAKE, dt=1, st=0, n=10, B=8, cnt=FAKE, g=None, grad=FAKE + 4096, gst=0):
        return lib.lib.mlpmoe_route_backward(x, dt, st, n, B, None, None, cnt, g, grad, gst, None)

    assert back(n=0) == lib.MLPMOE_OK
    for kw in (dict(x=None), dict(dt=2), dict(st=7), dict(gst=7), dict(n=-1), dict(B=0), dict(cnt=None), dict(grad=None), dict(g=FAKE + 1),
               dict(grad=FAKE + 2), dict(grad=FAKE, st=16, gst=8)):
        assert back(**kw) == bad, kw
    assert back(B=257) == lib.MLPMOE_ERR_UNSUPPORTED


def test_w4_quantize_refusals(lib):
    bad = lib.MLPMOE_ERR_INVALID_ARG

    def call(W=FAKE, dt=0, lay=1, st=0, rows=16, cols=64, g=32, q=FAKE, s=FAKE, z=FAKE):
        a = lib.lib.mlpmoe_w4_quantize(W, dt, lay, st, rows, cols, g, q, s, z, None)
        b = lib.lib.mlpmoe_w4_dequantize(q, s, z, rows, cols, g, W, dt, lay, st, None)
        assert a == b
        return a

    assert call(rows=0) == lib.MLPMOE_OK and call(cols=0) == lib.MLPMOE_OK
    for kw in (dict(W=None), dict(q=None), dict(s=None), dict(dt=2), dict(lay=2), dict(st=63), dict(lay=0, st=15), dict(rows=-1), dict(cols=-1),
               dict(q=FAKE + 8), dict(s=FAKE + 2), dict(z=FAKE + 1), dict(W=FAKE + 1)):
        assert call(**kw) == bad, kw
    for kw in (dict(g=16), dict(g=0), dict(g=256), dict(rows=(1 << 20) + 1), dict(cols=(1 << 20) + 1)):
        assert call(**kw) == lib.MLPMOE_ERR_UNSUPPORTED, kw


def test_w4_forward_refusals(lib):
    m = (FAKE, FAKE, None)

    def layer(d=64, I=64, d_b=(32, 32), group=32, gate=m, up=m, down=m):
        return lib.mlpmoe_w4_layer(d, I, list(d_b), group, gate, up, down)

    good = layer()
    size = lib.mlpmoe_w4_workspace(good, 5)
    bad = lib.MLPMOE_ERR_INVALID_ARG

    def call(l=good, x=FAKE, xt=0, xs=0, sc=None, xg=0, res=None, y=FAKE, yt=1, n=5, w=FAKE, wb=size):
        return lib.lib.mlpmoe_w4_forward(l, x, xt, xs, sc, xg, None, 1, res, y, yt, n, w, wb, None)

    assert call(n=0, x=None, y=None, w=None) == lib.MLPMOE_OK
    for kw in (dict(l=None), dict(x=None), dict(y=None), dict(xt=3), dict(yt=2), dict(xs=56), dict(xs=68), dict(xt=2), dict(xt=2, sc=FAKE, xg=48),
               dict(x=FAKE + 8), dict(y=FAKE + 4), dict(res=FAKE + 4), dict(res=FAKE, yt=0), dict(n=-1), dict(w=None), dict(wb=size - 1),
               dict(w=FAKE + 64), dict(xt=2, sc=FAKE + 2)):
        assert call(**kw) == bad, kw
    assert call(n=65537) == lib.MLPMOE_ERR_UNSUPPORTED
    assert call(l=layer(group=64), xt=2, sc=FAKE, xg=32) == lib.MLPMOE_ERR_UNSUPPORTED      # scales finer than the weights' groups
    part = lib.MLPMOE_ERR_BAD_PARTITION
    for l, want in ((layer(d_b=(32, 16)), part), (layer(d_b=(40, 24)), part), (layer(d_b=(64, 0)), part), (layer(d=60), lib.MLPMOE_ERR_UNSUPPORTED),
                    (layer(group=16), lib.MLPMOE_ERR_UNSUPPORTED), (layer(I=257 * 16, d_b=[16] * 257), lib.MLPMOE_ERR_UNSUPPORTED),
                    (layer(gate=(None, FAKE, None)), bad), (layer(up=(FAKE, None, None)), bad), (layer(down=(FAKE + 8, FAKE, None)), bad),
                    (layer(down=(FAKE, FAKE, FAKE + 8)), bad), (layer(d=0), bad)):
        assert call(l=l) == want
        with pytest.raises(lib.MlpmoeError):
            lib.mlpmoe_w4_workspace(l, 5)


def test_w4_workspace_grows_with_the_tokens(lib):
    m = (FAKE, FAKE, None)
    l = lib.mlpmoe_w4_layer(896, 4864, [304] * 16, 64, m, m, m)
    sizes = [lib.mlpmoe_w4_workspace(l, n) for n in (0, 1, 8, 9, 64, 65, 1000, 65536)]
    assert all(a <= b for a, b in zip(sizes, sizes[1:]))
    # the intermediate activations in fp32
    assert sizes[4] >= 64 * 4 * 4864


def test_w4_forward_has_kernels_for_every_documented_size(lib):
    """Every size is accepted with the workspace that is asked for: without a device a call gets as far as its first launch."""
    if torch.cuda.is_available():
        pytest.skip("the addresses here are not a device's")
    m = (FAKE, FAKE, FAKE)
    sizes = (8, 128, 1032, 14336, 48, 51328, 53248, 65520, 65536)
    for group in (32, 64, 128):
        for d in sizes:
            for I in sizes:
                for B in (1, 64, 256):
                    if I % 16 or I < 16 * B:
                        continue
                    layer = lib.mlpmoe_w4_layer(d, I, [16] * (B - 1) + [I - 16 * (B - 1)], group, m, m, m)
                    most = lib.mlpmoe_w4_workspace(layer, 64)
                    last = 0
                    for n in (1, 2, 3, 8, 9, 64):
                        size = lib.mlpmoe_w4_workspace(layer, n)
                        assert last <= size <= most              # a workspace serves any call of fewer tokens
                        last = size
                        for yt in (lib.MLPMOE_BF16, lib.MLPMOE_FP32):
                            for select in (None, FAKE):
                                rc = lib.lib.mlpmoe_w4_forward(layer, FAKE, 0, 0, None, 0, select, 1, None, FAKE, yt, n, FAKE, size, None)
                                assert rc == lib.MLPMOE_ERR_CUDA, (group, d, I, B, n, yt, select)


def test_binding_takes_buffers_and_streams_only(lib):
    """What is no buffer raises before the library is called; addresses and streams may be subclasses of int."""
    class Address(int):
        pass

    array, tensor = np.zeros(4, np.float32), torch.zeros(4)
    assert lib._ptr(None) is None and lib._ptr(Address(FAKE)) == FAKE
    assert lib._ptr(array) == array.ctypes.data and lib._ptr(tensor) == tensor.data_ptr()
    for wrong in (1.5, "4096", b"4096", [1, 2], np.float32(3.0), object()):
        with pytest.raises(AttributeError):
            lib._ptr(wrong)
        with pytest.raises(AttributeError):
            lib.mlpmoe_add_rmsnorm(wrong, None, None, None, 0, 64)
    assert lib._stream(None) is None and lib._stream(Address(7)) == 7
    for wrong in (1.5, "0"):
        with pytest.raises(AttributeError):
            lib._stream(wrong)
