"""GPU parity of the operators around a routed layer step with their float64 oracle: the residual norm with its 8-bit
output, the router with its balance loss and gradient, 4-bit weights and the layer on them; then a run of them together,
captured replays, side streams, guarded buffers and offsets past 32 bits.  Tolerances are derived beside each test
(u = 2^-24, half a step of fp32; bf16 2^-8, e4m3 2^-4 relative)."""
import numpy as np
import pytest
import torch

import oracle
from tests.helpers import Guarded, stream_ptr

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TORCH = {"bf16": torch.bfloat16, "fp32": torch.float32, "e4m3": torch.float8_e4m3fn}


def kind(lib, name):
    return {"bf16": lib.MLPMOE_BF16, "fp32": lib.MLPMOE_FP32, "e4m3": lib.MLPMOE_E4M3}[name]


def dev(a, name="fp32"):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda().to(TORCH[name])


def host(t):
    return t.float().cpu().numpy().astype(np.float64)


def strided(a, name, pad):
    """The rows of `a` on the device, `pad` elements of NaN behind each (nothing may use them)."""
    n, d = a.shape
    full = torch.full((n, d + pad), float("nan"), dtype=torch.float32)
    full[:, :d] = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32))
    return full.cuda().to(TORCH[name])[:, :d]


# ------------------------------------------------------------------------------------------------ residual norm

NORM_CASES = [
    # n, d, x, r, out, group, pad
    (1, 1, "fp32", "fp32", "fp32", 0, 0), (1, 4096, "fp32", "bf16", "bf16", 0, 0), (3, 7, "bf16", "none", "e4m3", 0, 1), (5, 8, "fp32", "bf16", "e4m3", 32, 8),
    (2, 33, "fp32", "fp32", "e4m3", 32, 0), (297, 896, "fp32", "bf16", "e4m3", 128, 0), (300, 1000, "bf16", "bf16", "e4m3", 64, 8),
    (301, 1001, "bf16", "fp32", "fp32", 0, 3), (298, 1032, "fp32", "none", "bf16", 0, 0), (299, 4095, "fp32", "bf16", "e4m3", 128, 0),
    (310, 4096, "bf16", "bf16", "e4m3", 0, 16), (2, 4104, "fp32", "bf16", "e4m3", 128, 0), (1, 8192, "fp32", "fp32", "bf16", 0, 0),
    (2, 8200, "bf16", "fp32", "e4m3", 128, 0), (2, 20001, "fp32", "bf16", "fp32", 0, 0), (1, 32768, "fp32", "bf16", "e4m3", 0, 0), (4, 100, "fp32", "fp32", "e4m3", 128, 28),
    (4100, 512, "fp32", "bf16", "e4m3", 128, 0), (4099, 100, "bf16", "fp32", "bf16", 0, 3), (4098, 264, "fp32", "bf16", "e4m3", 64, 8),
    (1030, 4096, "fp32", "bf16", "e4m3", 128, 0), (1029, 2057, "bf16", "fp32", "e4m3", 64, 3), (300, 2048, "fp32", "bf16", "e4m3", 32, 0),
]


@pytest.mark.parametrize("n,d,xt,rt,ot,group,pad", NORM_CASES)
@pytest.mark.parametrize("inplace", [False, True])
def test_add_rmsnorm(lib, n, d, xt, rt, ot, group, pad, inplace):
    rng = np.random.default_rng([d, n, group])
    x = strided(rng.normal(size=(n, d)) * np.exp(rng.normal(size=(n, 1))), xt, pad)
    r = None if rt == "none" else strided(rng.normal(size=(n, d)), rt, pad)
    if n > 2:
        x[1] = 0
        if r is not None:
            r[1] = 0                                        # a row of zeros
    gain = dev(1 + 0.2 * rng.normal(size=d))
    xs, rs = host(x), None if r is None else host(r)
    s, v = oracle.add_rmsnorm(xs, rs, host(gain))
    out = Guarded((n, d), TORCH[ot])
    x_out = None if inplace else Guarded((n, d), TORCH[xt])
    ng = -(-d // (group or d))
    scales = Guarded((n, ng), torch.float32)
    lib.mlpmoe_add_rmsnorm(x, r, x if inplace else x_out.t, out.t, n, d, gain=gain, scales=scales.t if ot == "e4m3" else None, group=group,
                           x_dtype=kind(lib, xt), r_dtype=kind(lib, "fp32" if r is None else rt), out_dtype=kind(lib, ot), x_stride=x.stride(0),
                           r_stride=0 if r is None else r.stride(0), x_out_stride=x.stride(0) if inplace else 0, stream=stream_ptr())
    torch.cuda.synchronize()
    out.check()
    scales.check()
    # one fp32 addition, then bf16's rounding where x is bf16: the same bits as here
    want = xs.astype(np.float32) if rs is None else xs.astype(np.float32) + rs.astype(np.float32)
    got = host(x if inplace else x_out.t)
    assert np.array_equal(got, oracle.round_to_bf16(want) if xt == "bf16" else want.astype(np.float64))
    if not inplace:
        x_out.check()
    elif pad:
        base = torch.as_strided(x, (n, d + pad), (d + pad, 1))
        assert bool(torch.isnan(base[:, d:].float()).all())            # what stands behind the rows is left alone
    # the sum of squares: a thread adds up to 32 terms, then 5 shuffles and up to 32 partial sums: 70 roundings of
    # positive terms, halved by the root; s itself 2 u; division, root, reciprocal and two products 6 u
    rel = 45 * U
    got = host(out.t)
    if ot != "e4m3":
        assert np.all(np.abs(got - v) <= (rel + (2.0 ** -8 if ot == "bf16" else 0.0)) * np.abs(v) + 1e-38)
        return
    _, sc = oracle.quantize_e4m3(v, group)
    got_sc = host(scales.t)
    assert np.all(np.abs(got_sc - sc) <= (rel + U) * sc)
    per = np.repeat(got_sc, group or d, axis=1)[:, :d]
    # half a step of e4m3 (2^-4 of the value, 2^-10 of the scale below 2^-6), on a value that is rel off
    assert np.all(np.abs(got * per - v) <= np.maximum(2.0 ** -4 * np.abs(v), 2.0 ** -10 * per) * (1 + 2.0 ** -12) + (rel + 4 * U) * np.abs(v))
    if n > 2:
        assert np.all(got[1] == 0) and np.all(got_sc[1] == np.float32(2.0 ** -126))


def test_add_rmsnorm_without_gain_and_without_x_out(lib):
    rng = np.random.default_rng(5)
    x, r = dev(rng.normal(size=(9, 264))), dev(rng.normal(size=(9, 264)), "bf16")
    keep = x.clone()
    out = torch.empty(9, 264, device="cuda")
    lib.mlpmoe_add_rmsnorm(x, r, None, out, 9, 264, r_dtype=lib.MLPMOE_BF16, out_dtype=lib.MLPMOE_FP32, eps=1e-3, stream=stream_ptr())
    _, v = oracle.add_rmsnorm(host(keep), host(r), None, 1e-3)
    assert torch.equal(x, keep) and np.all(np.abs(host(out) - v) <= 45 * U * np.abs(v))
    # the plain norm of the library: the same operator without its additions
    plain = torch.empty(9, 264, device="cuda")
    lib.mlpmoe_rmsnorm(keep, plain, 9, 264, 1e-3, lib.MLPMOE_FP32, stream_ptr())
    lib.mlpmoe_add_rmsnorm(keep, None, None, out, 9, 264, out_dtype=lib.MLPMOE_FP32, eps=1e-3, stream=stream_ptr())
    assert np.all(np.abs(host(out) - host(plain)) <= 90 * U * np.abs(host(plain)))


# ------------------------------------------------------------------------------------------------ router

def run_route(lib, logits, k, dtype, avail=None, valid=None, grad_loss=None):
    n, B = logits.shape
    sel, cnt = Guarded((max(n, 1), B), torch.uint8), Guarded((B + 1,), torch.int32)
    prob, loss, grad = Guarded((B,), torch.float32), Guarded((1,), torch.float32), Guarded((max(n, 1), B), TORCH[dtype])
    size = lib.mlpmoe_route_workspace(n, B)
    ws = Guarded((size,), torch.uint8)
    lib.mlpmoe_route(logits, n, B, k, sel.t, cnt.t, prob.t, loss.t, ws.t, size, dtype=kind(lib, dtype), stride=logits.stride(0) if n else 0,
                     avail=avail, valid=valid, stream=stream_ptr())
    lib.mlpmoe_route_backward(logits, cnt.t, grad.t, n, B, grad_loss=grad_loss, dtype=kind(lib, dtype), stride=logits.stride(0) if n else 0,
                              avail=avail, valid=valid, stream=stream_ptr())
    torch.cuda.synchronize()
    for b in (sel, cnt, prob, loss, grad, ws):
        b.check()
    return sel.t, cnt.t, prob.t, loss.t, grad.t


def check_route(lib, values, k, dtype, pad=0, avail=None, valid=None, g=None):
    logits = strided(values, dtype, pad)
    lh = host(logits)
    n, B = lh.shape
    da = None if avail is None else torch.from_numpy(np.asarray(avail, np.uint8)).cuda()
    dv = None if valid is None else torch.from_numpy(np.asarray(valid, np.uint8)).cuda()
    dg = None if g is None else dev([g])
    sel, cnt, prob, loss, grad = run_route(lib, logits, k, dtype, da, dv, dg)
    r = oracle.route(lh, k, avail, valid)
    assert np.array_equal(sel.cpu().numpy()[:n], r["select"])
    assert np.array_equal(cnt.cpu().numpy(), r["counts"])
    # a probability: x - max is rounded once (u of at most `span`), expf is good to 2 ulp, the row's sum is at most 8 + 5
    # additions of positive terms, then a reciprocal and a product; a column's sum adds up to 600 of them in all
    span = float(np.nanmax(np.where(np.isfinite(lh), lh, np.nan)) - np.nanmin(np.where(np.isfinite(lh), lh, np.nan))) if np.isfinite(lh).any() else 0.0
    span = min(span, 104.0)                                # below that expf is 0 in fp32 (1e-45 absolute)
    rel = (span + 4 + 13 + 3) * U
    assert np.all(np.abs(host(prob) - r["prob"]) <= (rel + 600 * U) * r["prob"] + 1e-38)
    assert abs(float(loss) - r["loss"]) <= (rel + 604 * U) * r["loss"] + 1e-38
    want, size = oracle.route_grad(lh, r["counts"], avail, valid, 1.0 if g is None else g)
    # two terms, each a product of two such factors and a dot product of B positive terms; then the type's rounding
    tol = (2 * rel + (B + 20) * U) * size + (2.0 ** -8 if dtype == "bf16" else 0.0) * np.abs(want) + 1e-38
    assert np.all(np.abs(host(grad)[:n] - want) <= tol)
    return r


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n,B,k", [(1, 1, 1), (1, 2, 1), (3, 5, 5), (17, 8, 2), (64, 16, 4), (65, 31, 7), (129, 32, 8), (1000, 64, 16), (77, 100, 3),
                                   (513, 128, 16), (40, 129, 9), (300, 256, 256), (5000, 13, 2)])
def test_route_and_gradient(lib, n, B, k, dtype):
    rng = np.random.default_rng([n, B, k])
    values = np.round(rng.normal(size=(n, B)) * 2 * 16) / 16          # coarse: ties in most rows
    check_route(lib, values, k, dtype, pad=0)
    avail = (rng.uniform(size=B) < 0.7).astype(np.uint8)
    avail[rng.integers(B)] = 1
    valid = (rng.uniform(size=n) < 0.8).astype(np.uint8)
    # places and rows that are masked hold NaN and infinities; live places may hold -infinity
    values = values.copy()
    values[rng.uniform(size=(n, B)) < 0.1] = -np.inf
    for bad in (np.nan, np.inf):
        values[:, avail == 0] = np.where(rng.uniform(size=(n, int((avail == 0).sum()))) < 0.5, bad, values[:, avail == 0])
    values[valid == 0] = np.nan
    check_route(lib, values, k, dtype, pad=4 if B % 4 == 0 else 3, avail=avail, valid=valid, g=-1.5)


def test_route_rows_with_nothing(lib):
    values = np.full((4, 6), -np.inf)
    r = check_route(lib, values, 3, "fp32")
    assert r["loss"] == 0 and r["counts"].sum() == 0
    check_route(lib, np.zeros((4, 6)), 3, "bf16", avail=np.zeros(6, np.uint8))
    check_route(lib, np.zeros((4, 6)), 3, "fp32", valid=np.zeros(4, np.uint8))
    values[2, 4] = 1.0
    values[1, 0], values[1, 5] = np.nan, -3.0
    r = check_route(lib, values, 3, "fp32")
    assert r["counts"].tolist() == [0, 0, 0, 0, 1, 1, 2]


def test_route_extreme_logits(lib):
    big = float(np.finfo(np.float32).max)
    values = np.array([[big, -big, 0.0, big], [-0.0, 0.0, -0.0, 1e-45], [-big, -big, -big, -big], [np.inf, 0.0, np.inf, 1.0]])
    sel, cnt, prob, loss, grad = run_route(lib, dev(values), 2, "fp32")
    r = oracle.route(values, 2)
    assert np.array_equal(sel.cpu().numpy(), [[1, 0, 0, 1], [1, 0, 0, 1], [1, 1, 0, 0], [1, 0, 1, 0]])
    assert np.allclose(host(prob), r["prob"], rtol=100 * U, atol=0) and np.isclose(float(loss), r["loss"], rtol=1e-6)
    assert bool(torch.isfinite(grad).all())


def test_route_of_no_tokens_clears_its_sums(lib):
    cnt, prob, loss = torch.full((9,), 7, device="cuda", dtype=torch.int32), torch.ones(8, device="cuda"), torch.ones(1, device="cuda")
    size = lib.mlpmoe_route_workspace(0, 8)
    ws = torch.empty(size, device="cuda", dtype=torch.uint8)
    lib.mlpmoe_route(None, 0, 8, 2, None, cnt, prob, loss, ws, size, stream=stream_ptr())
    lib.mlpmoe_route_backward(None, cnt, None, 0, 8, stream=stream_ptr())
    assert int(cnt.abs().sum()) == 0 and float(prob.sum()) == 0 and float(loss) == 0


def test_route_gradient_in_place_and_same_bits(lib):
    rng = np.random.default_rng(8)
    logits = dev(rng.normal(size=(3000, 48)))
    a = run_route(lib, logits, 6, "fp32")
    b = run_route(lib, logits, 6, "fp32")
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    same = logits.clone()
    lib.mlpmoe_route_backward(same, a[1], same, 3000, 48, stream=stream_ptr())
    assert torch.equal(same, a[4])


# ------------------------------------------------------------------------------------------------ 4-bit weights

def pack_dev(codes, scales, zeros, asym, pad=15):
    q, s, z = oracle.w4_pack(codes, scales, zeros, pad)
    return (torch.from_numpy(q).cuda(), torch.from_numpy(s).cuda().to(torch.bfloat16), torch.from_numpy(z).cuda() if asym else None)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,cols,group,asym", [(1, 1, 32, True), (8, 8, 128, False), (16, 64, 32, False), (33, 100, 32, True), (40, 257, 64, True),
                                                  (24, 130, 128, False), (65, 1000, 128, True), (100, 96, 64, False)])
def test_w4_quantize_and_back(lib, rows, cols, group, asym, dtype):
    rng = np.random.default_rng([rows, cols, group])
    W = rng.normal(size=(rows, cols)).astype(np.float32) * 0.02
    if rows > 3:
        W[1], W[2], W[3] = 0.0, np.abs(W[2]) + 0.5, W[3] * 1e-30
    for paper in (False, True):
        for pad in (0, 5):
            src = W.T if paper else W
            w = strided(src, dtype, pad)
            wh = host(w).astype(np.float32)
            codes, scales, zeros = oracle.w4_quantize(wh.T if paper else wh, group, asym)
            ng, r16 = scales.shape[0], -(-rows // 16) * 16
            q, s = Guarded((rows, -(-cols // 32) * 16), torch.uint8), Guarded((ng, r16), torch.bfloat16)
            z = Guarded((ng, r16), torch.uint8) if asym else None
            s.t.fill_(-1.0)
            layout = lib.MLPMOE_LAYOUT_PAPER if paper else lib.MLPMOE_LAYOUT_LINEAR
            lib.mlpmoe_w4_quantize(w, rows, cols, group, q.t, s.t, z.t if asym else None, dtype=kind(lib, dtype), layout=layout,
                                   stride=w.stride(0), stream=stream_ptr())
            # scales are bf16(range / 7 | 15) and codes rint of an fp32 quotient, all correctly rounded: equal bits
            assert np.array_equal(oracle.w4_unpack(q.t.cpu().numpy(), rows, cols), codes)
            assert np.array_equal(host(s.t)[:, :rows], scales) and np.all(host(s.t)[:, rows:] == -1)
            if asym:
                assert np.array_equal(z.t.cpu().numpy()[:, :rows], zeros)
                z.check()
            q.check()
            s.check()
            want = oracle.w4_dequantize(codes, scales, zeros, group)
            for out in ("fp32", "bf16"):
                back = strided(np.zeros_like(src), out, pad)
                lib.mlpmoe_w4_dequantize(q.t, s.t, z.t if asym else None, rows, cols, group, back, dtype=kind(lib, out), layout=layout,
                                         stride=back.stride(0), stream=stream_ptr())
                got = host(back)
                exact = want if out == "fp32" else oracle.round_to_bf16(want)      # at most 13 significant bits: exact in fp32
                assert np.array_equal(got.T if paper else got, exact)


def test_w4_quantize_smallest_and_largest_ranges(lib):
    """Scales at and below the smallest normal number (a reciprocal past fp32's range), and a range that overflows."""
    rng = np.random.default_rng(91)
    W = rng.uniform(-1, 1, size=(48, 128)).astype(np.float32)
    W *= (2.0 ** np.repeat(np.arange(-132, -116), 3))[:, None].astype(np.float32)
    for dtype in ("fp32", "bf16"):
        for asym in (False, True):
            w = dev(W, dtype)
            codes, scales, zeros = oracle.w4_quantize(host(w).astype(np.float32), 64, asym)
            assert (scales == 0).any() and (scales > 0).any()
            q, s = torch.empty(48, 64, device="cuda", dtype=torch.uint8), torch.empty(2, 48, device="cuda", dtype=torch.bfloat16)
            z = torch.empty(2, 48, device="cuda", dtype=torch.uint8) if asym else None
            lib.mlpmoe_w4_quantize(w, 48, 128, 64, q, s, z, dtype=kind(lib, dtype), stream=stream_ptr())
            assert np.array_equal(oracle.w4_unpack(q.cpu().numpy(), 48, 128), codes) and np.array_equal(host(s), scales)
            assert not asym or np.array_equal(z.cpu().numpy(), zeros)
    big = torch.full((1, 32), 3e38, device="cuda")
    big[0, 1] = -3e38
    q, s, z = torch.empty(1, 16, device="cuda", dtype=torch.uint8), torch.empty(1, 16, device="cuda", dtype=torch.bfloat16), torch.empty(1, 16, device="cuda", dtype=torch.uint8)
    lib.mlpmoe_w4_quantize(big, 1, 32, 32, q, s, z, dtype=lib.MLPMOE_FP32, stream=stream_ptr())
    assert float(s[0, 0]) == float("inf") and int(z[0, 0]) == 0 and int(q.max()) == 0


def test_w4_quantize_halves_go_to_even(lib):
    """Every quotient of bf16 significands that lies half way between two whole numbers, and its neighbours."""
    div = np.arange(128, 256)
    for asym in (False, True):
        top = 15 if asym else 7
        rows = []
        for b in div:
            half = (np.arange(0 if asym else -7, top) + 0.5) * b
            near = np.concatenate([half - 1, half - 0.5, half, half + 0.5, half + 1])
            near = near[near == oracle.round_to_bf16(near)]
            near = near[(np.abs(near) <= top * b) & ((near >= 0) if asym else True)][:127]
            rows.append(np.concatenate([[top * b], near, np.zeros(127 - len(near))]))
        W = np.array(rows, dtype=np.float32)
        W[:, 0] = oracle.round_to_bf16(W[:, 0])
        for dtype in ("bf16", "fp32"):
            w = dev(W, dtype)
            codes, scales, zeros = oracle.w4_quantize(host(w).astype(np.float32), 128, asym)
            q, s = torch.empty(128, 64, device="cuda", dtype=torch.uint8), torch.empty(1, 128, device="cuda", dtype=torch.bfloat16)
            z = torch.empty(1, 128, device="cuda", dtype=torch.uint8) if asym else None
            lib.mlpmoe_w4_quantize(w, 128, 128, 128, q, s, z, dtype=kind(lib, dtype), stream=stream_ptr())
            assert np.array_equal(oracle.w4_unpack(q.cpu().numpy(), 128, 128), codes) and np.array_equal(host(s), scales)


class W4Case:
    """A layer on 4-bit weights with garbage in every padding, and its oracle."""

    def __init__(self, lib, key, d, d_b, group, asym, alpha=None, std=0.2):
        rng = np.random.default_rng(key)
        self.lib, self.d, self.I, self.d_b, self.group, self.alpha = lib, d, sum(d_b), list(d_b), group, alpha
        self.W, self.mats = [], []
        for rows, cols in ((self.I, d), (self.I, d), (d, self.I)):
            codes, scales, zeros = oracle.w4_quantize(rng.normal(size=(rows, cols)) * std, group, asym)
            if not asym:
                codes[rng.uniform(size=codes.shape) < 0.01] = 0          # the code -8, which the quantiser does not make
            self.W.append(oracle.w4_dequantize(codes, scales, zeros, group))
            self.mats.append(pack_dev(codes, scales, zeros, asym))
        self.layer = lib.mlpmoe_w4_layer(d, self.I, self.d_b, group, *self.mats, alpha=alpha)

    def activations(self, key, n, xt, x_group=0):
        """(host values, tensor, scales)"""
        rng = np.random.default_rng(key)
        x = rng.normal(size=(n, self.d))
        if xt != "e4m3":
            t = strided(x, xt, 8)
            return host(t), t, None
        codes, scales = oracle.quantize_e4m3(x, x_group)
        sc = scales.astype(np.float32)
        return codes * np.repeat(sc.astype(np.float64), x_group or self.d, axis=1)[:, :self.d], strided(codes, "e4m3", 16 - self.d % 16), dev(sc)

    def run(self, x, n, xt, yt, scales=None, x_group=0, select=None, compensate=True, residual=None, stream=None):
        lib = self.lib
        size = lib.mlpmoe_w4_workspace(self.layer, n)
        ws, y = Guarded((size,), torch.uint8), Guarded((n, self.d), TORCH[yt])
        lib.mlpmoe_w4_forward(self.layer, x, y.t, n, ws.t, size, x_dtype=kind(lib, xt), x_stride=x.stride(0), x_scale=scales, x_group=x_group,
                              select=select, compensate=compensate, residual=residual, y_dtype=kind(lib, yt),
                              stream=stream_ptr() if stream is None else stream)
        torch.cuda.synchronize()
        ws.check()
        y.check()
        return y.t

    def tolerance(self, r, xh, yt, fp16=None):
        """Inside a group of K the activations are whole multiples of a unit, a power of two of which the group's largest is at
        least 2^22 / 1.004 (y fp32) or 2^14 / 1.004 (y bf16): off by half a unit, 1.004 * 2^-23 or 1.004 * 2^-15 of it.  The
        products are exact.  Sums in fp32: one term per group and digit, up to 16 + 8 parts to join, and six roundings of a
        term (scale times unit, the product, a factor for e4m3's scale); the digits of x add up to at most 3 |x| in magnitude.
        fp16 (the type of x): the tensor-core kernels, which hold a value as fp16 times a unit that brings the largest of its
        row or block of 128 to 2^14 at least: off by 2^-11 of the value (x in bf16: not at all) or half of 2^-24 units,
        2^-39 of the largest; a group's products are added in fp32, in any order."""
        q = 1.004 * (2.0 ** -23 if yt == "fp32" else 2.0 ** -15)
        starts = np.arange(0, self.d, self.group)
        top = np.maximum.reduceat(np.abs(xh), starts, axis=1)
        terms = 30
        if fp16:
            q, terms = 2.0 ** -39, 30 + self.group
            top = np.broadcast_to(np.abs(xh).max(axis=1, keepdims=True), top.shape)

        def product(K, size, tops, W, starts, each):
            return (3 * U * (K / self.group + terms) + each) * size + q * (tops @ np.add.reduceat(np.abs(W), starts, axis=1).T)
        each = 2.0 ** -11 if fp16 and fp16 != "bf16" else 0.0
        e_gate, e_up = product(self.d, r["abs_gate"], top, self.W[0], starts, each), product(self.d, r["abs_up"], top, self.W[1], starts, each)
        # |silu'| <= 1.1; expf, the quotient and the two products cost 2^-20 of h (and |g| u from the exponent)
        h_err = np.abs(r["alpha"]) * (1.1 * e_gate * (np.abs(r["up"]) + e_up) + np.abs(oracle.silu(r["gate"])) * e_up)
        h_err = np.where(r["on"], h_err, 0.0) + (2.0 ** -20 + np.abs(r["gate"]) * 2 * U) * np.abs(r["h"])
        starts = np.arange(0, self.I, self.group)
        tops = np.maximum.reduceat(np.abs(r["h"]) + h_err, starts, axis=1)
        size = np.abs(r["h"]) @ np.abs(self.W[2]).T
        if fp16:                                           # a block of 128 holds its groups
            blocks = np.maximum.reduceat(tops, np.arange(0, tops.shape[1], 128 // self.group), axis=1)
            tops = np.repeat(blocks, 128 // self.group, axis=1)[:, :tops.shape[1]]
        each = 2.0 ** -11 if fp16 else 0.0
        return r["coef"][:, None] * (h_err @ np.abs(self.W[2]).T + product(self.I, size, tops, self.W[2], starts, each)) + 4 * U * np.abs(r["y"])

    def check(self, y, xh, xt, yt, select=None, compensate=True, residual=None, fp16=False):
        r = oracle.w4_layer_forward(xh, *self.W, self.d_b, self.alpha, select, compensate, residual)
        tol = self.tolerance(r, xh, yt, xt if fp16 else None)
        if residual is not None:
            tol = tol + 2 * U * np.abs(np.asarray(residual, dtype=np.float64))
        if yt == "bf16":
            tol = tol + 2.0 ** -8 * np.abs(r["y"])
        got = host(y)
        assert np.all(np.isfinite(got)) and np.all(np.abs(got - r["y"]) <= tol + 1e-30)
        return r


@pytest.mark.parametrize("group,asym", [(32, False), (32, True), (64, True), (64, False), (128, False), (128, True)])
@pytest.mark.parametrize("n", [1, 2, 3, 8, 9, 17, 22, 33, 64, 65, 131])
def test_w4_forward_tokens(lib, n, group, asym):
    c = W4Case(lib, [group, asym], 328, [48, 16, 208, 64], group, asym, alpha=[1.0, -0.5, 0.8, 1.2])
    for xt, yt in (("bf16", "fp32"), ("fp32", "bf16"), ("fp32", "fp32"), ("bf16", "bf16")):
        xh, x, _ = c.activations([n, 1], n, xt)
        c.check(c.run(x, n, xt, yt), xh, xt, yt)


@pytest.mark.parametrize("d,d_b", [(8, [16]), (16, [16, 16]), (40, [16, 32]), (136, [16] * 9), (256, [512]), (904, [64, 1200]), (1032, [2048, 16])])
@pytest.mark.parametrize("group", [32, 128])
def test_w4_forward_sizes(lib, d, d_b, group):
    c = W4Case(lib, [d, group], d, d_b, group, True)
    for n, xt, yt in ((1, "bf16", "fp32"), (5, "bf16", "bf16"), (40, "fp32", "fp32")):
        xh, x, _ = c.activations([n, d], n, xt)
        residual = np.random.default_rng(n).normal(size=(n, d)).astype(np.float32)
        c.check(c.run(x, n, xt, yt, residual=dev(residual)), xh, xt, yt, residual=residual)


@pytest.mark.parametrize("group,x_group", [(32, 0), (32, 32), (32, 64), (32, 128), (64, 64), (64, 128), (128, 128), (128, 0)])
def test_w4_forward_e4m3(lib, group, x_group):
    c = W4Case(lib, [group, x_group], 424, [112, 160], group, False)
    for n in (1, 9, 65):
        xh, x, sc = c.activations([n, 2], n, "e4m3", x_group)
        c.check(c.run(x, n, "e4m3", "fp32", sc, x_group), xh, "e4m3", "fp32")


@pytest.mark.parametrize("n", [1, 6, 70])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_w4_forward_selection(lib, n, group):
    """Tokens on some branches, on none, on all; branches nobody takes (their weights hold NaN scales: they must not be
    read into a result); branches with alpha = 0; with and without compensation."""
    d_b = [16, 48, 128, 16, 256, 96, 112, 64]
    c = W4Case(lib, [n, group], 200, d_b, group, True, alpha=[1.0, 0.7, 0.0, -1.1, 1.0, 0.9, 1.3, 1.0])
    xh, x, _ = c.activations([n, 3], n, "bf16")
    rng = np.random.default_rng([n, 4])
    sel = (rng.uniform(size=(n, 8)) < 0.4).astype(np.uint8)
    sel[:, 4] = 0                                          # nobody
    sel[:, 2] = 1                                          # everybody, but its alpha is 0
    if n > 2:
        sel[1], sel[2] = 0, 255                            # no branch; every branch (any non-zero byte selects)
        sel[:, 4] = 0
    ds = torch.from_numpy(sel).cuda()
    residual = rng.normal(size=(n, 200)).astype(np.float32)
    for comp in (True, False):
        for yt in ("fp32", "bf16"):
            r = c.check(c.run(x, n, "bf16", yt, select=ds, compensate=comp, residual=dev(residual)), xh, "bf16", yt, sel, comp, residual)
    # a branch that no token computes is not read: NaN scales there change nothing
    off = oracle.branch_offsets(d_b)
    gate_scale = c.mats[0][1].clone()
    c.mats[0][1][:, off[4]:off[5]] = float("nan")
    c.mats[0][1][:, off[2]:off[3]] = float("nan")
    c.check(c.run(x, n, "bf16", "fp32", select=ds, residual=dev(residual)), xh, "bf16", "fp32", sel, True, residual)
    # without a selection: the branch with alpha = 0 stays out, the others are all computed
    c.mats[0][1].copy_(gate_scale)
    c.mats[0][1][:, off[2]:off[3]] = float("nan")
    c.check(c.run(x, n, "bf16", "fp32"), xh, "bf16", "fp32")
    # no token selects anything
    none = torch.zeros(n, 8, device="cuda", dtype=torch.uint8)
    assert torch.equal(c.run(x, n, "bf16", "fp32", select=none, residual=dev(residual)), dev(residual))


@pytest.mark.parametrize("group,asym", [(32, True), (64, False), (128, True)])
def test_w4_forward_tensor_core_kernels(lib, group, asym):
    """Layers large enough, with enough tokens and y in bf16, for the kernels of the 5th-generation tensor cores: ragged
    d_model and d_inter, every type of x, chunks of one token less and more than they hold, selections."""
    d, d_b = 1032, [1008, 7040, 16, 3008, 4944]
    c = W4Case(lib, [group, 7], d, d_b, group, asym, alpha=[1.0, 0.7, 1.2, -0.6, 0.9], std=0.05)
    rng = np.random.default_rng([group, 8])
    for n, xt, x_group in ((17, "bf16", 0), (33, "fp32", 0), (64, "bf16", 0), (65, "bf16", 0), (40, "e4m3", 128), (130, "e4m3", 0)):
        xh, x, sc = c.activations([n, 9], n, xt, x_group)
        residual = rng.normal(size=(n, d)).astype(np.float32)
        c.check(c.run(x, n, xt, "bf16", sc, x_group, residual=dev(residual)), xh, xt, "bf16", residual=residual, fp16=True)
        sel = (rng.uniform(size=(n, 5)) < 0.4).astype(np.uint8)
        sel[:, 3], sel[0] = 0, 0
        for comp in (True, False):
            c.check(c.run(x, n, xt, "bf16", sc, x_group, select=torch.from_numpy(sel).cuda(), compensate=comp), xh, xt, "bf16", sel, comp, fp16=True)
    none = torch.zeros(130, 5, device="cuda", dtype=torch.uint8)
    assert float(c.run(x, 130, "e4m3", "bf16", sc, 0, select=none).abs().max()) == 0
    # alpha = 0 drops a branch without a selection; what it holds does not matter
    c.alpha = [1.0, 0.0, 1.2, -0.6, 0.9]
    c.layer = lib.mlpmoe_w4_layer(d, c.I, d_b, group, *c.mats, alpha=c.alpha)
    c.mats[0][1][:, 1008:8048] = float("nan")
    xh, x, _ = c.activations([64, 9], 64, "bf16")
    c.check(c.run(x, 64, "bf16", "bf16"), xh, "bf16", "bf16", fp16=True)


def test_w4_forward_wait_limit(lib):
    """A wait inside the tensor cores' kernels that runs out: the call returns, the status says so, and the next call is
    right again."""
    d, d_b = 1032, [4512, 4496]
    c = W4Case(lib, [55], d, d_b, 128, False, std=0.05)
    xh, x, _ = c.activations([56], 64, "bf16")
    size = lib.mlpmoe_w4_workspace(c.layer, 64)
    ws, y = torch.empty(size, device="cuda", dtype=torch.uint8), torch.empty(64, d, device="cuda", dtype=torch.bfloat16)

    def call():
        lib.mlpmoe_w4_forward(c.layer, x, y, 64, ws, size, x_stride=x.stride(0), y_dtype=lib.MLPMOE_BF16, stream=stream_ptr())
        return lib.mlpmoe_w4_get_status(ws, stream_ptr())
    assert call() == lib.MLPMOE_OK
    c.check(y, xh, "bf16", "bf16", fp16=True)
    lib.mlpmoe_w4_debug_set_wait(20_000_000, 1)
    try:
        assert call() == lib.MLPMOE_ERR_DEVICE_TIMEOUT
    finally:
        lib.mlpmoe_w4_debug_set_wait()
    y.zero_()
    assert call() == lib.MLPMOE_OK
    c.check(y, xh, "bf16", "bf16", fp16=True)
    # the other kernels have no such waits and report so
    lib.mlpmoe_w4_forward(c.layer, x, y, 3, ws, size, x_stride=x.stride(0), y_dtype=lib.MLPMOE_BF16, stream=stream_ptr())
    assert lib.mlpmoe_w4_get_status(ws, stream_ptr()) == lib.MLPMOE_OK


# paths of the layer's kernels: (d_model, branch widths, tokens, type of y)
PATHS = {"stream": (520, [96, 160, 256], 5, "fp32"), "tiled": (520, [96, 160, 256], 40, "fp32"), "tensor": (1032, [4512, 16, 4480], 66, "bf16")}


@pytest.mark.parametrize("path", list(PATHS))
def test_w4_forward_graphs_and_streams(lib, path):
    """Two captured calls with a workspace each, replayed on new inputs from two streams at once, give the eager call's bits;
    so do eager calls from two streams."""
    d, d_b, n, yt = PATHS[path]
    c = W4Case(lib, [61], d, d_b, 64, True, std=0.05)
    size = lib.mlpmoe_w4_workspace(c.layer, n)
    xs = [dev(np.random.default_rng([62, i]).normal(size=(n, d)), "bf16") for i in range(4)]
    want = [c.run(x, n, "bf16", yt).clone() for x in xs]
    side = [torch.cuda.Stream() for _ in range(2)]
    x_in = [xs[0].clone(), xs[1].clone()]
    ws = [torch.empty(size, device="cuda", dtype=torch.uint8) for _ in range(2)]
    y = [torch.empty(n, d, device="cuda", dtype=TORCH[yt]) for _ in range(2)]
    graphs = []
    torch.cuda.synchronize()
    for k in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side[k]):
            lib.mlpmoe_w4_forward(c.layer, x_in[k], y[k], n, ws[k], size, y_dtype=kind(lib, yt), stream=stream_ptr())
        graphs.append(g)
    for first in (0, 2):
        for k in range(2):
            x_in[k].copy_(xs[first + k])
            y[k].zero_()
        torch.cuda.synchronize()
        for _ in range(10):
            for k in range(2):
                with torch.cuda.stream(side[k]):
                    graphs[k].replay()
        torch.cuda.synchronize()
        for k in range(2):
            assert torch.equal(y[k], want[first + k])
    for _ in range(10):
        for k in range(2):
            lib.mlpmoe_w4_forward(c.layer, xs[k], y[k], n, ws[k], size, y_dtype=kind(lib, yt), stream=side[k].cuda_stream)
    torch.cuda.synchronize()
    assert torch.equal(y[0], want[0]) and torch.equal(y[1], want[1])
    del graphs


@pytest.mark.parametrize("path", list(PATHS))
@pytest.mark.parametrize("stored", [(True, False, False), (False, True, True), (False, False, True)])
def test_w4_forward_zeros_stored_for_some_matrices(lib, path, stored):
    """zero = NULL beside matrices that have zeros."""
    d, d_b, n, yt = PATHS[path]
    c = W4Case(lib, [63, *stored], d, d_b, 32, True, std=0.05)
    for k, keep in enumerate(stored):
        if not keep:                                       # the codes stay: the weights move by (zero - 8) * scale
            q, s, z = c.mats[k]
            rows, cols = c.W[k].shape
            codes = oracle.w4_unpack(q.cpu().numpy(), rows, cols)
            scales = host(s)[:, :rows]
            c.W[k] = oracle.w4_dequantize(codes, scales, np.full(scales.shape, 8, np.uint8), 32)
            c.mats[k] = (q, s, None)
    c.layer = lib.mlpmoe_w4_layer(d, c.I, d_b, 32, *c.mats)
    xh, x, _ = c.activations([64], n, "bf16")
    c.check(c.run(x, n, "bf16", yt), xh, "bf16", yt, fp16=path == "tensor")


@pytest.mark.parametrize("path", list(PATHS))
def test_w4_forward_padded_batch(lib, path):
    """Tokens that select nothing may hold anything (NaN, infinities): their rows are the residual, the others are not touched."""
    d, d_b, n, yt = PATHS[path]
    c = W4Case(lib, [65], d, d_b, 128, False, std=0.05)
    xh, x, _ = c.activations([66], n, "bf16")
    sel = np.ones((n, len(d_b)), np.uint8)
    sel[::2, 0], sel[n - 2:] = 0, 0
    x[n - 2], x[n - 1] = float("nan"), float("inf")
    xh[n - 2:] = 0.0
    residual = np.random.default_rng(67).normal(size=(n, d)).astype(np.float32)
    y = c.run(x, n, "bf16", yt, select=torch.from_numpy(sel).cuda(), residual=dev(residual))
    c.check(y, xh, "bf16", yt, sel, True, residual, fp16=path == "tensor")
    assert torch.equal(y[n - 2:], dev(residual)[n - 2:].to(y.dtype))


@pytest.mark.parametrize("path", list(PATHS))
def test_w4_forward_magnitudes(lib, path):
    """Tokens of very different magnitude in one call, a token of zeros, and one whose values span 2^20."""
    d, d_b, n, yt = PATHS[path]
    c = W4Case(lib, [68], d, d_b, 64, True, std=0.05)
    rng = np.random.default_rng(69)
    xh = rng.normal(size=(n, d))
    xh[0], xh[1], xh[2], xh[3] = xh[0] * 1e6, xh[1] * 1e-6, 0.0, xh[3] * 2.0 ** rng.uniform(-20, 0, size=d)
    for xt in ("bf16", "fp32"):
        x = dev(xh, xt)
        c.check(c.run(x, n, xt, yt), host(x), xt, yt, fp16=path == "tensor")


@pytest.mark.parametrize("d,d_b", [(65536, [64, 80]), (128, [65520, 16])])
def test_w4_forward_longest_rows(lib, d, d_b):
    """The largest d_model and d_inter, on every path, all branches and a selection."""
    c = W4Case(lib, [73, d], d, d_b, 128, True, std=0.02)
    for n, yt, fp16 in ((1, "fp32", False), (8, "bf16", False), (11, "fp32", False), (40, "bf16", True)):
        xh, x, _ = c.activations([74, n], n, "bf16")
        c.check(c.run(x, n, "bf16", yt), xh, "bf16", yt, fp16=fp16)
        sel = np.zeros((n, 2), np.uint8)
        sel[:, 1] = 1
        c.check(c.run(x, n, "bf16", yt, select=torch.from_numpy(sel).cuda()), xh, "bf16", yt, sel, fp16=fp16)


def test_w4_forward_most_branches(lib):
    """256 branches of 16 neurons on every path, a selection of 8 per token."""
    d_b = [16] * 256
    rng = np.random.default_rng(70)
    for d, n, yt in ((136, 4, "bf16"), (136, 20, "fp32"), (1032, 72, "bf16")):
        c = W4Case(lib, [71, n], d, d_b, 32, False, std=0.05)
        xh, x, _ = c.activations([72, n], n, "bf16")
        sel = np.zeros((n, 256), np.uint8)
        for t in range(n):
            sel[t, rng.permutation(256)[:8]] = 1
        c.check(c.run(x, n, "bf16", yt, select=torch.from_numpy(sel).cuda()), xh, "bf16", yt, sel, fp16=n == 72)


def test_w4_forward_residual_in_place_and_same_bits(lib):
    c = W4Case(lib, [77], 512, [128] * 8, 64, False)
    xh, x, _ = c.activations([5], 12, "bf16")
    r0 = np.random.default_rng(6).normal(size=(12, 512)).astype(np.float32)
    size = lib.mlpmoe_w4_workspace(c.layer, 12)
    ws = torch.empty(size, device="cuda", dtype=torch.uint8)
    ys = []
    for _ in range(3):
        y = dev(r0)
        lib.mlpmoe_w4_forward(c.layer, x, y, 12, ws, size, x_stride=x.stride(0), residual=y, stream=stream_ptr())
        ys.append(y)
        ws.fill_(0xFF)                                     # nothing is kept in the workspace from call to call
    assert torch.equal(ys[0], ys[1]) and torch.equal(ys[0], ys[2])
    c.check(ys[0], xh, "bf16", "fp32", residual=r0)


@pytest.mark.parametrize("d,I,n,yt", [(896, 4864, 1, "fp32"), (896, 4864, 13, "fp32"), (4096, 14336, 1, "fp32"), (4096, 14336, 64, "fp32"),
                                      (4096, 14336, 64, "bf16")])
def test_w4_forward_full_size(lib, d, I, n, yt):
    """The Qwen- and Llama-shaped layers against float64 on the device, on weights that the library quantised itself."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(d + n)
    group, mats, deq = 128, [], []
    for rows, cols in ((I, d), (I, d), (d, I)):
        W = (torch.randn(rows, cols, device="cuda", generator=gen) * 0.02).bfloat16()
        q = torch.empty(rows, cols // 2, device="cuda", dtype=torch.uint8)
        s = torch.empty(cols // group, rows, device="cuda", dtype=torch.bfloat16)
        z = torch.empty(cols // group, rows, device="cuda", dtype=torch.uint8)
        lib.mlpmoe_w4_quantize(W, rows, cols, group, q, s, z, stream=stream_ptr())
        back = torch.empty(rows, cols, device="cuda")
        lib.mlpmoe_w4_dequantize(q, s, z, rows, cols, group, back, dtype=lib.MLPMOE_FP32, stream=stream_ptr())
        mats.append((q, s, z))
        deq.append(back.double())
        # half a step of at most range / 15 and the roundings of scale and zero
        assert float((back - W.float()).abs().max()) <= 0.02 * 12 / 15
    x = torch.randn(n, d, device="cuda", generator=gen).bfloat16()
    layer = lib.mlpmoe_w4_layer(d, I, [I // 16] * 16, group, *mats)
    size = lib.mlpmoe_w4_workspace(layer, n)
    ws, y = torch.empty(size, device="cuda", dtype=torch.uint8), torch.empty(n, d, device="cuda", dtype=TORCH[yt])
    lib.mlpmoe_w4_forward(layer, x, y, n, ws, size, y_dtype=kind(lib, yt), stream=stream_ptr())
    xd = x.double()
    g, u = xd @ deq[0].t(), xd @ deq[1].t()
    h = torch.nn.functional.silu(g) * u
    # as W4Case.tolerance, on the device
    q = 1.004 * (2.0 ** -23 if yt == "fp32" else 2.0 ** -15)

    def product(K, size, v, W):
        tops = v.abs().view(n, -1, group).amax(2)
        return 3 * U * (K / group + 30) * size + q * (tops @ W.abs().view(W.shape[0], -1, group).sum(2).t())
    eg, eu = (product(d, xd.abs() @ w.abs().t(), xd, w) for w in deq[:2])
    h_err = 1.1 * eg * (u.abs() + eu) + torch.nn.functional.silu(g).abs() * eu + (2.0 ** -20 + g.abs() * 2 * U) * h.abs()
    size_y = h.abs() @ deq[2].abs().t()
    if yt == "bf16" and n == 64 and d == 4096:             # the tensor-core kernels: h in fp16, a group's sum in fp32
        h_err = h_err + 2.0 ** -11 * h.abs() + 3 * U * group * h.abs()
    tol = h_err @ deq[2].abs().t() + product(I, size_y, h.abs() + h_err, deq[2]) + (4 * U + (2.0 ** -8 if yt == "bf16" else 0)) * (h @ deq[2].t()).abs() + 1e-30
    assert bool(((y.double() - h @ deq[2].t()).abs() <= tol).all())


# ------------------------------------------------------------------------------------------------ together

def test_a_routed_decode_step(lib):
    """residual norm -> router -> layer on the selection -> residual norm, as a decode step calls them: eagerly, on a side
    stream, and captured into a graph that is replayed on new inputs; with 8-bit activations between norm and layer."""
    d, d_b, n, B, k, group = 256, [64, 16, 176, 128], 7, 4, 2, 64
    c = W4Case(lib, [99], d, d_b, group, True, alpha=[1.0, 0.9, 1.1, 0.7], std=0.08)
    rng = np.random.default_rng(10)
    router = rng.normal(size=(d, B)) * 0.2
    gain = 1 + 0.1 * rng.normal(size=d)
    dr, dg = dev(router), dev(gain)
    x, r = torch.empty(n, d, device="cuda"), torch.empty(n, d, device="cuda", dtype=torch.bfloat16)
    xo, out, sc = torch.empty_like(x), torch.empty(n, d, device="cuda", dtype=torch.float8_e4m3fn), torch.empty(n, d // group, device="cuda")
    logits, sel = torch.empty(n, B, device="cuda"), torch.empty(n, B, device="cuda", dtype=torch.uint8)
    cnt, prob, loss = torch.empty(B + 1, device="cuda", dtype=torch.int32), torch.empty(B, device="cuda"), torch.empty(1, device="cuda")
    y, x2, out2 = torch.empty(n, d, device="cuda", dtype=torch.bfloat16), torch.empty_like(x), torch.empty(n, d, device="cuda", dtype=torch.bfloat16)
    rs, ws = lib.mlpmoe_route_workspace(n, B), lib.mlpmoe_w4_workspace(c.layer, n)
    rw, ww = torch.empty(rs, device="cuda", dtype=torch.uint8), torch.empty(ws, device="cuda", dtype=torch.uint8)

    def step():
        st = stream_ptr()
        lib.mlpmoe_add_rmsnorm(x, r, xo, out, n, d, gain=dg, scales=sc, group=group, r_dtype=lib.MLPMOE_BF16, out_dtype=lib.MLPMOE_E4M3, stream=st)
        torch.mm(out.float() * sc.repeat_interleave(group, 1), dr, out=logits)
        lib.mlpmoe_route(logits, n, B, k, sel, cnt, prob, loss, rw, rs, stream=st)
        lib.mlpmoe_w4_forward(c.layer, out, y, n, ww, ws, x_dtype=lib.MLPMOE_E4M3, x_scale=sc, x_group=group, select=sel, y_dtype=lib.MLPMOE_BF16, stream=st)
        lib.mlpmoe_add_rmsnorm(xo, y, x2, out2, n, d, r_dtype=lib.MLPMOE_BF16, stream=st)

    def load(seed):
        g = np.random.default_rng(seed)
        x.copy_(dev(g.normal(size=(n, d))))
        r.copy_(dev(g.normal(size=(n, d)), "bf16"))

    def check():
        torch.cuda.synchronize()
        s, v = oracle.add_rmsnorm(host(x), host(r), gain)
        xh = host(out) * np.repeat(host(sc), group, axis=1)
        assert np.all(np.abs(xh - v) <= np.maximum(2.0 ** -4 * np.abs(v), 2.0 ** -10 * np.repeat(host(sc), group, axis=1)) * (1 + 1e-3))
        lo = oracle.route(host(logits), k)
        assert np.array_equal(sel.cpu().numpy(), lo["select"]) and np.array_equal(cnt.cpu().numpy(), lo["counts"])
        c.check(y, xh, "e4m3", "bf16", sel.cpu().numpy())
        s2, v2 = oracle.add_rmsnorm(host(xo), host(y))
        assert np.all(np.abs(host(x2) - s2) <= U * np.abs(s2)) and np.all(np.abs(host(out2) - v2) <= (2.0 ** -8 + 45 * U) * np.abs(v2))

    load(1)
    step()
    check()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        load(2)
        step()
    torch.cuda.current_stream().wait_stream(side)
    check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (3, 4, 5):
        load(seed)
        for b in (ww, rw):
            b.fill_(0xFF)
        graph.replay()
        check()
    del graph


def test_router_feeds_the_routed_forward(lib):
    """mlpmoe_route's selection is what mlpmoe_forward_routed takes (a layer of the library with a pruned branch: the router
    is told by `avail`), and w4_dequantize's weights make a layer that mlpmoe_create takes."""
    d, d_b, n, B, group = 256, [64, 128, 64, 128], 300, 4, 128
    c = W4Case(lib, [101], d, d_b, group, False, std=0.05)
    dense = []
    for (q, s, z), rows, cols in zip(c.mats, (c.I, c.I, d), (d, d, c.I)):
        W = torch.empty(rows, cols, device="cuda", dtype=torch.bfloat16)
        lib.mlpmoe_w4_dequantize(q, s, z, rows, cols, group, W, stream=stream_ptr())
        dense.append(W)
    h = lib.mlpmoe_create(d, c.I, d_b, *dense, None, lib.MLPMOE_BF16, lib.MLPMOE_LAYOUT_LINEAR, n, stream_ptr())
    try:
        lib.mlpmoe_prune(h, [True, False, True, True], True, stream_ptr())
        rng = np.random.default_rng(11)
        xh, x, _ = c.activations([12], n, "bf16")
        x = x.contiguous()
        logits = dev(rng.normal(size=(n, B)))
        avail = torch.tensor([1, 0, 1, 1], device="cuda", dtype=torch.uint8)
        sel, cnt, *_ = run_route(lib, logits, 2, "fp32", avail)
        y = torch.empty(n, d, device="cuda")
        lib.mlpmoe_forward_routed(h, x, y, n, sel, True, stream_ptr())
        torch.cuda.synchronize()
        alpha = [float(np.float32(a)) for a in oracle.prune_alpha([1.0] * 4, [True, False, True, True])]
        host_w = [host(w) for w in dense]
        ref = oracle.routed_forward(xh, host_w[0].T, host_w[1].T, host_w[2].T, d_b, alpha, sel.cpu().numpy())
        assert np.max(np.abs(host(y) - ref)) <= 2e-2 * np.sqrt(np.mean(ref ** 2))
        assert cnt.cpu().tolist()[1] == 0
        # the same step on the 4-bit weights themselves, a pass of 64 tokens at a time
        c4 = lib.mlpmoe_w4_layer(d, c.I, d_b, group, *c.mats, alpha=alpha)
        c.alpha, c.layer = alpha, c4
        c.check(c.run(x, n, "bf16", "fp32", select=sel), xh, "bf16", "fp32", sel.cpu().numpy())
    finally:
        lib.mlpmoe_destroy(h)


def test_router_training_steps(lib):
    """Descending the gradient through the library's forward and backward makes an unbalanced router's gradient steps run:
    finite, zero row sums, and equal to the differences of the loss at constant counts."""
    rng = np.random.default_rng(13)
    logits = dev(rng.normal(size=(64, 8)) + np.linspace(0, 2, 8))
    for _ in range(3):
        sel, cnt, prob, loss, grad = run_route(lib, logits, 2, "fp32")
        lh, ch = host(logits), cnt.cpu().numpy()
        f = ch[:-1] / ch[:-1].sum()
        direction = rng.normal(size=lh.shape)

        def value(e):
            return 8 * float(np.dot(f, oracle.route(lh + e * direction, 2)["p"].sum(axis=0) / ch[-1]))
        want = (value(1e-4) - value(-1e-4)) / 2e-4
        # the gradient's own bound (see check_route) against the direction, and the differences' 1e-8
        assert abs(float(np.sum(host(grad) * direction)) - want) <= 1e-4 * np.abs(host(grad) * direction).sum() + 1e-7
        logits = logits - 5.0 * grad


# ------------------------------------------------------------------------------------------------ long offsets

def test_rows_past_32_bit_offsets(lib):
    """Rows 2^30 + 8 elements apart: offsets past 2^32 bytes and past 2^31 elements."""
    stride, n, d = (1 << 30) + 8, 4, 64
    rng = np.random.default_rng(14)
    big = torch.empty(stride * (n - 1) + d, device="cuda", dtype=torch.bfloat16)
    rows = torch.as_strided(big, (n, d), (stride, 1))
    rows.copy_(dev(rng.normal(size=(n, d)), "bf16"))
    out = torch.empty(n, d, device="cuda")
    lib.mlpmoe_add_rmsnorm(rows, None, None, out, n, d, x_dtype=lib.MLPMOE_BF16, out_dtype=lib.MLPMOE_FP32, x_stride=stride, stream=stream_ptr())
    _, v = oracle.add_rmsnorm(host(rows))
    assert np.all(np.abs(host(out) - v) <= 45 * U * np.abs(v))
    sel, cnt, prob, loss, _ = run_route(lib, rows, 3, "bf16")
    r = oracle.route(host(rows), 3)
    assert np.array_equal(sel.cpu().numpy(), r["select"])
    c = W4Case(lib, [15], d, [32, 16], 32, False)
    c.check(c.run(rows, n, "bf16", "fp32"), host(rows), "bf16", "fp32")
