"""GPU parity of the operators of a training step around a routed layer with their float64 oracle: the sorted order, rows to their
branches and back with the gradient, LayerNorm and the norms' gradient, AdamW; then a step of them together, captured replays and
offsets past 32 bits.  Tolerances are derived beside each test (u = 2^-24, half a step of fp32; bf16 2^-8, e4m3 2^-4 relative)."""
import numpy as np
import pytest
import torch

import oracle
from tests.helpers import POISON, Guarded, stream_ptr
from tests.test_gpu_operators import TORCH, U, dev, host, kind, strided

pytestmark = pytest.mark.gpu

BF16 = 2.0 ** -8
TINY = 2.0 ** -149          # what fp32 cannot hold


def ints(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def selection(rng, n, B, mean, empty=True):
    """A uint8 mask with about `mean` branches a token; some tokens select nothing, some many, any value but 0 selects."""
    select = (rng.uniform(size=(n, B)) < min(1.0, mean / B)).astype(np.uint8) * rng.integers(1, 256, (n, B)).astype(np.uint8)
    if empty and n > 3:
        select[1] = 0
        select[2] = 255
        if B > 2:
            select[:, 1] = 0             # a branch that nobody selects
    return select


class Plan:
    """mlpmoe_sort_tokens of a selection on the device, and the oracle's."""

    def __init__(self, lib, select, slots, align, offset=0):
        n, B = select.shape
        self.want = oracle.sort_tokens(select, slots, align)
        self.n, self.B, self.slots, self.align = n, B, slots, align
        self.used = len(self.want["row_token"])
        self.rows = max(1, lib.mlpmoe_sort_rows(n, B, slots, align))
        raw = torch.zeros(n * B + 64, dtype=torch.uint8, device="cuda")
        raw[offset:offset + n * B] = torch.from_numpy(select.reshape(-1)).cuda()
        self.select = raw[offset:offset + n * B]
        i32 = torch.int32
        self.offsets, self.counts, self.row_token = Guarded((B + 1,), i32), Guarded((B,), i32), Guarded((self.rows,), i32)
        self.token_row, self.token_branch = Guarded((max(n, 1), slots), i32), Guarded((max(n, 1), slots), i32)
        self.row_token.t.view(torch.uint8).fill_(POISON)
        size = lib.mlpmoe_sort_workspace(n, B)
        self.work = Guarded((size,), torch.uint8)
        self.run(lib)

    def run(self, lib, stream=None):
        lib.mlpmoe_sort_tokens(self.select, self.n, self.B, self.slots, self.offsets.t, self.counts.t, self.row_token.t, self.rows, self.token_row.t,
                               self.work.t, self.work.nbytes, align=self.align, token_branch=self.token_branch.t,
                               stream=stream_ptr() if stream is None else stream)

    def check(self):
        torch.cuda.synchronize()
        for name in ("offsets", "counts", "token_row", "token_branch"):
            buffer = getattr(self, name)
            buffer.check()
            assert np.array_equal(buffer.t.cpu().numpy()[:self.n] if name.startswith("token") else buffer.t.cpu().numpy(), self.want[name]), name
        got = self.row_token.t.cpu().numpy()
        assert np.array_equal(got[:self.used], self.want["row_token"])
        assert np.all(got[self.used:].view(np.uint8) == POISON)              # rows behind the last branch are left alone
        self.row_token.check()
        self.work.check()


# ------------------------------------------------------------------------------------------------ the sorted order

@pytest.mark.parametrize("n,B,slots,align,mean", [
    (0, 3, 2, 1, 1), (1, 1, 1, 1, 1), (1, 256, 256, 1024, 9), (2, 5, 3, 8, 2), (31, 16, 4, 1, 3), (33, 5, 2, 1, 2), (64, 16, 4, 8, 4), (1000, 31, 31, 1, 6),
    (1024, 128, 8, 128, 8), (512, 256, 5, 1, 5), (513, 256, 300, 16, 20), (1025, 33, 16, 4, 7), (5000, 100, 7, 1024, 4), (4099, 32, 40, 1, 30),
    (129, 40, 3, 8, 4), (160, 256, 9, 128, 9), (1025, 32, 8, 1, 8), (1056, 128, 4, 2, 4), (2048, 256, 8, 64, 8), (2049, 129, 8, 1, 8), (30001, 256, 3, 16, 2), (40000, 7, 2, 1, 1), (200000, 4, 2, 128, 2), (530001, 3, 2, 1, 1)])
def test_sort_tokens(lib, n, B, slots, align, mean):
    Plan(lib, selection(np.random.default_rng([n, B]), n, B, mean), slots, align).check()


@pytest.mark.parametrize("n,B", [(100, 32), (100, 12), (2000, 48), (2000, 20)])
@pytest.mark.parametrize("offset", [1, 2, 4, 8])
def test_sort_tokens_of_unaligned_masks(lib, n, B, offset):
    Plan(lib, selection(np.random.default_rng(n + B), n, B, 4), 6, 4, offset).check()


def test_sort_tokens_of_nothing_and_of_everything(lib):
    for n in (5, 3000):
        Plan(lib, np.zeros((n, 40), np.uint8), 3, 64).check()
        Plan(lib, np.ones((n, 40), np.uint8), 40, 64).check()
        Plan(lib, np.ones((n, 40), np.uint8), 1, 1).check()


def test_sort_tokens_again_and_without_branches(lib):
    select = selection(np.random.default_rng(7), 3000, 24, 5)
    plan = Plan(lib, select, 6, 8)
    plan.check()
    plan.work.t.fill_(0xEE)                              # nothing of the last call is needed
    plan.run(lib)
    plan.check()
    keep = plan.token_branch.t.clone()
    plan.token_branch.t.fill_(5)
    lib.mlpmoe_sort_tokens(plan.select, 3000, 24, 6, plan.offsets.t, plan.counts.t, plan.row_token.t, plan.rows, plan.token_row.t, plan.work.t,
                           plan.work.nbytes, align=8, stream=stream_ptr())
    torch.cuda.synchronize()
    assert bool((plan.token_branch.t == 5).all())
    plan.token_branch.t.copy_(keep)
    plan.check()


# ------------------------------------------------------------------------------------------------ rows to their branches and back

MOVES = [
    # n, B, slots, align, d, pad of the rows
    (1, 1, 1, 1, 1, 0), (1, 4, 2, 8, 4096, 0), (5, 3, 3, 1, 7, 1), (33, 8, 4, 16, 896, 0), (70, 16, 4, 1, 264, 8), (65, 33, 5, 4, 1000, 3), (64, 40, 40, 1, 136, 0),
    (300, 12, 2, 128, 520, 0), (130, 9, 3, 2, 4097, 0), (40, 6, 2, 32, 8200, 8), (37, 5, 2, 1, 257, 0), (20, 4, 2, 4, 511, 2), (9, 3, 3, 1, 3, 0),
    (50, 6, 6, 1, 2, 1), (31, 4, 2, 8, 256, 1), (29, 4, 2, 1, 1023, 4)]


@pytest.mark.parametrize("n,B,slots,align,d,pad", MOVES)
@pytest.mark.parametrize("dtype,group", [("fp32", 0), ("bf16", 0), ("e4m3", 0), ("e4m3", 32), ("e4m3", 128)])
def test_dispatch(lib, n, B, slots, align, d, pad, dtype, group):
    rng = np.random.default_rng([n, d])
    plan = Plan(lib, selection(rng, n, B, slots), slots, align)
    x = strided(rng.normal(size=(n, d)), dtype, pad)
    rows = Guarded((plan.rows, d + pad), TORCH[dtype])
    rows.t.view(torch.uint8).fill_(POISON)
    ng = -(-d // (group or d))
    scale = dev(rng.uniform(0.1, 1, (n, ng))) if dtype == "e4m3" else None
    row_scale = Guarded((plan.rows, ng), torch.float32)
    row_scale.t.view(torch.uint8).fill_(POISON)
    lib.mlpmoe_dispatch(x, rows.t, n, d, B, slots, plan.offsets.t, plan.counts.t, plan.token_row.t, plan.rows, align=align, dtype=kind(lib, dtype),
                        x_scale=scale, row_scale=row_scale.t if scale is not None else None, group=group, x_stride=x.stride(0), rows_stride=d + pad,
                        stream=stream_ptr())
    torch.cuda.synchronize()
    rows.check()
    row_scale.check()
    es = x.element_size()
    got = rows.t.view(torch.uint8).view(plan.rows, -1).cpu().numpy()
    src = x.contiguous().view(torch.uint8).view(n, -1).cpu().numpy()
    token = plan.want["row_token"]
    assert np.array_equal(got[:plan.used, :d * es], np.where(token[:, None] >= 0, src[token], 0))
    assert np.all(got[plan.used:] == POISON) and np.all(got[:, d * es:] == POISON)
    if scale is not None:
        assert np.array_equal(host(row_scale.t)[:plan.used], np.where(token[:, None] >= 0, host(scale)[token], 0.0))
    assert np.all(row_scale.t.view(torch.uint8).view(plan.rows, -1).cpu().numpy()[plan.used if scale is not None else 0:] == POISON)


@pytest.mark.parametrize("n,B,slots,align,d,pad", MOVES)
@pytest.mark.parametrize("rt,st,yt,weighted", [("bf16", "fp32", "fp32", True), ("fp32", "none", "fp32", True), ("bf16", "bf16", "bf16", True),
                                               ("fp32", "fp32", "bf16", False), ("bf16", "none", "fp32", False)])
def test_combine(lib, n, B, slots, align, d, pad, rt, st, yt, weighted):
    rng = np.random.default_rng([n, d, 1])
    plan = Plan(lib, selection(rng, n, B, slots), slots, align)
    rows = strided(rng.normal(size=(plan.rows, d)), rt, pad)
    rows[plan.used:] = float("nan")                              # what belongs to no branch is not read
    token_row = plan.want["token_row"]
    w = np.where(token_row >= 0, rng.normal(size=(n, slots)), np.nan)      # nor are the weights of places without a row
    weight = dev(w) if weighted else None
    res = None if st == "none" else strided(rng.normal(size=(n, d)) * 3, st, pad)
    y = Guarded((n, d + pad), TORCH[yt])
    y.t.view(torch.uint8).fill_(POISON)
    lib.mlpmoe_combine(rows, plan.rows, plan.token_row.t, slots, y.t, n, d, weight=weight, residual=res, rows_dtype=kind(lib, rt),
                       residual_dtype=kind(lib, "fp32" if res is None else st), y_dtype=kind(lib, yt), rows_stride=rows.stride(0),
                       residual_stride=0 if res is None else res.stride(0), y_stride=d + pad, stream=stream_ptr())
    torch.cuda.synchronize()
    y.check()
    rows64, w64 = host(rows), np.nan_to_num(host(weight)) if weighted else None
    want = oracle.combine(rows64, token_row, w64, None if res is None else host(res))
    size = oracle.combine(np.abs(np.nan_to_num(rows64)), token_row, None if w64 is None else np.abs(w64), None if res is None else np.abs(host(res)))
    # a product and a sum of at most `slots` terms and the residual: one rounding each
    bound = (slots + 2) * U * size + (BF16 * np.abs(want) if yt == "bf16" else 0.0) + TINY
    assert np.all(np.abs(host(y.t[:, :d]) - want) <= bound)
    if pad:
        assert bool((y.t[:, d:].contiguous().view(torch.uint8) == POISON).all())


@pytest.mark.parametrize("n,B,slots,align,d,pad", MOVES + [(3, 2, 2, 1, 20001, 0), (2, 3, 2, 8, 32768, 0), (9, 64, 50, 1, 300, 0)])
@pytest.mark.parametrize("gt,rt,weighted", [("fp32", "bf16", True), ("bf16", "bf16", True), ("fp32", "fp32", True), ("bf16", "fp32", False)])
@pytest.mark.parametrize("inplace", [False, True])
def test_combine_backward(lib, n, B, slots, align, d, pad, gt, rt, weighted, inplace):
    rng = np.random.default_rng([n, d, 2])
    plan = Plan(lib, selection(rng, n, B, slots), slots, align)
    gy = strided(rng.normal(size=(n, d)), gt, pad)
    rows = strided(rng.normal(size=(plan.rows, d)), rt, pad)
    token_row = plan.want["token_row"]
    weight = dev(np.where(token_row >= 0, rng.normal(size=(n, slots)), np.nan)) if weighted else None
    rows64, gy64, w64 = host(rows), host(gy), np.nan_to_num(host(weight)) if weighted else None
    grad_rows = torch.full_like(torch.as_strided(rows, (plan.rows, d + pad), (d + pad, 1)), 7.0)
    out = rows if inplace else grad_rows
    grad_w = Guarded((n, slots), torch.float32)
    lib.mlpmoe_combine_backward(gy, rows, plan.rows, plan.token_row.t, slots, out, grad_w.t, n, d, weight=weight, B=B, align=align,
                                offsets=plan.offsets.t, counts=plan.counts.t, grad_y_dtype=kind(lib, gt), rows_dtype=kind(lib, rt),
                                grad_y_stride=gy.stride(0), rows_stride=rows.stride(0), grad_rows_stride=d + pad, stream=stream_ptr())
    torch.cuda.synchronize()
    grad_w.check()
    want_rows, want_w = oracle.combine_grad(gy64, rows64, token_row, w64)
    got = host(out[:, :d])
    # one product, and bf16's rounding
    assert np.all(np.abs(got - want_rows)[:plan.used] <= (U + (BF16 if rt == "bf16" else 0.0)) * (1 + BF16) * np.abs(want_rows)[:plan.used] + TINY)
    assert np.array_equal(got[plan.used:], rows64[plan.used:] if inplace else np.full((plan.rows - plan.used, d), 7.0))
    if pad and not inplace:
        assert bool((grad_rows[:, d:] == 7.0).all())
    _, size = oracle.combine_grad(np.abs(gy64), np.abs(rows64), token_row)
    # a thread adds up to 64 products, then 5 shuffles and up to 32 warps
    assert np.all(np.abs(host(grad_w.t) - want_w) <= 102 * U * size)


def test_combine_backward_of_one_of_the_two(lib):
    rng = np.random.default_rng(11)
    plan = Plan(lib, selection(rng, 50, 6, 2), 2, 4)
    gy, rows, w = dev(rng.normal(size=(50, 264))), dev(rng.normal(size=(plan.rows, 264))), dev(rng.normal(size=(50, 2)))
    both_r, both_w = torch.full_like(rows, 7.0), torch.empty(50, 2, device="cuda")
    args = dict(weight=w, B=6, align=4, offsets=plan.offsets.t, counts=plan.counts.t, rows_dtype=lib.MLPMOE_FP32, stream=stream_ptr())
    lib.mlpmoe_combine_backward(gy, rows, plan.rows, plan.token_row.t, 2, both_r, both_w, 50, 264, **args)
    only_r, only_w = torch.full_like(rows, 7.0), torch.empty(50, 2, device="cuda")
    lib.mlpmoe_combine_backward(gy, None, plan.rows, plan.token_row.t, 2, only_r, None, 50, 264, **args)
    lib.mlpmoe_combine_backward(gy, rows, plan.rows, plan.token_row.t, 2, None, only_w, 50, 264, **args)
    assert torch.equal(both_r, only_r) and torch.equal(both_w, only_w)


def test_places_outside_of_the_rows_are_skipped(lib):
    rng = np.random.default_rng(12)
    place = ints([[0, 5], [9, -7], [3, 2147483647]])
    rows, x = Guarded((5, 40), torch.float32), dev(rng.normal(size=(3, 40)))
    rows.t.fill_(7.0)
    lib.mlpmoe_dispatch(x, rows.t, 3, 40, 1, 2, None, None, place, 5, dtype=lib.MLPMOE_FP32, stream=stream_ptr())
    want = np.full((5, 40), 7.0)
    want[0], want[3] = host(x)[0], host(x)[2]
    assert np.array_equal(host(rows.t), want)
    rows.check()
    y = torch.empty(3, 40, device="cuda")
    lib.mlpmoe_combine(rows.t, 5, place, 2, y, 3, 40, rows_dtype=lib.MLPMOE_FP32, stream=stream_ptr())
    assert np.array_equal(host(y), np.stack((want[0], np.zeros(40), want[3])))
    grad_w = torch.empty(3, 2, device="cuda")
    lib.mlpmoe_combine_backward(x, rows.t, 5, place, 2, rows.t, grad_w, 3, 40, rows_dtype=lib.MLPMOE_FP32, stream=stream_ptr())
    rows.check()
    assert np.array_equal(host(rows.t), want) and np.array_equal(host(grad_w) != 0, [[True, False], [False, False], [True, False]])


def test_rows_that_are_not_finite_stay_with_their_tokens(lib):
    rng = np.random.default_rng(13)
    plan = Plan(lib, selection(rng, 40, 5, 2, empty=False), 2, 1)
    rows = rng.normal(size=(plan.rows, 72))
    token = plan.want["row_token"]
    bad = int(token[3])
    rows[3, 10] = np.inf
    y = torch.empty(40, 72, device="cuda")
    lib.mlpmoe_combine(dev(rows), plan.rows, plan.token_row.t, 2, y, 40, 72, rows_dtype=lib.MLPMOE_FP32, stream=stream_ptr())
    fine = np.isfinite(host(y))
    assert not fine[bad, 10] and fine.sum() == 40 * 72 - 1


# ------------------------------------------------------------------------------------------------ LayerNorm

LAYERS = [
    # n, d, x, r, out, group, pad
    (1, 1, "fp32", "fp32", "fp32", 0, 0), (1, 4096, "fp32", "bf16", "bf16", 0, 0), (3, 7, "bf16", "none", "e4m3", 0, 1), (5, 8, "fp32", "bf16", "e4m3", 32, 8),
    (297, 896, "fp32", "bf16", "e4m3", 128, 0), (301, 1001, "bf16", "fp32", "fp32", 0, 3), (298, 1032, "fp32", "none", "bf16", 0, 0),
    (310, 4096, "bf16", "bf16", "e4m3", 0, 16), (1, 8192, "fp32", "fp32", "bf16", 0, 0), (2, 8200, "bf16", "fp32", "e4m3", 128, 0),
    (2, 20001, "fp32", "bf16", "fp32", 0, 0), (1, 32768, "fp32", "bf16", "fp32", 0, 0), (4100, 512, "fp32", "bf16", "bf16", 0, 0),
    (4099, 100, "bf16", "fp32", "fp32", 0, 3), (1030, 4096, "fp32", "bf16", "e4m3", 128, 0), (300, 2057, "fp32", "bf16", "fp32", 0, 3),
    (77, 1001, "bf16", "bf16", "bf16", 0, 0), (50, 257, "bf16", "bf16", "bf16", 0, 2), (33, 1, "bf16", "bf16", "bf16", 0, 0), (40, 515, "bf16", "none", "bf16", 0, 1),
    (5000, 131, "bf16", "bf16", "bf16", 0, 0), (1100, 4095, "bf16", "bf16", "bf16", 0, 0)]


@pytest.mark.parametrize("n,d,xt,rt,ot,group,pad", LAYERS)
@pytest.mark.parametrize("inplace", [False, True])
def test_add_layernorm(lib, n, d, xt, rt, ot, group, pad, inplace):
    rng = np.random.default_rng([d, n, group, 1])
    x = strided(rng.normal(size=(n, d)) * np.exp(rng.normal(size=(n, 1))) + 0.3, xt, pad)
    r = None if rt == "none" else strided(rng.normal(size=(n, d)), rt, pad)
    if n > 2:
        x[1] = 0.5
        if r is not None:
            r[1] = -0.25                                    # a row of one value: its norm is the bias
    gain, bias = dev(1 + 0.2 * rng.normal(size=d)), dev(0.2 * rng.normal(size=d))
    xs, rs = host(x), None if r is None else host(r)
    s, v = oracle.add_layernorm(xs, rs, host(gain), host(bias))
    out, x_out = Guarded((n, d), TORCH[ot]), None if inplace else Guarded((n, d), TORCH[xt])
    scales = Guarded((n, -(-d // (group or d))), torch.float32)
    lib.mlpmoe_add_layernorm(x, r, x if inplace else x_out.t, out.t, n, d, gain=gain, bias=bias, scales=scales.t if ot == "e4m3" else None, group=group,
                             x_dtype=kind(lib, xt), r_dtype=kind(lib, "fp32" if r is None else rt), out_dtype=kind(lib, ot), x_stride=x.stride(0),
                             r_stride=0 if r is None else r.stride(0), x_out_stride=x.stride(0) if inplace else 0, stream=stream_ptr())
    torch.cuda.synchronize()
    out.check()
    scales.check()
    want = xs.astype(np.float32) if rs is None else xs.astype(np.float32) + rs.astype(np.float32)
    assert np.array_equal(host(x if inplace else x_out.t), oracle.round_to_bf16(want) if xt == "bf16" else want.astype(np.float64))
    # s: one rounding.  The mean: a sum of up to 32 terms a thread, 5 shuffles, 32 partial sums and the division, 70 u of mean |s|; z = s - mean
    # takes that, and 2 u of its own.  The squares' sum again 70 u, halved by the root, and what z is off by; root, reciprocal, products 6 u.
    mean_abs = np.abs(s).mean(axis=1, keepdims=True)
    z = s - s.mean(axis=1, keepdims=True)
    var = (z * z).mean(axis=1, keepdims=True)
    off = 70 * U * mean_abs + 2 * U * (np.abs(z) + np.abs(s))
    q = 1.0 / np.sqrt(var + 1e-5)
    rel = 41 * U + (np.abs(z) * off).mean(axis=1, keepdims=True) * q * q * 1.01 + (off * off).mean(axis=1, keepdims=True) * q * q
    bound = np.abs(host(gain)) * q * (off + np.abs(z) * rel) * 1.01 + 2 * U * (np.abs(v) + np.abs(host(bias)))
    got = host(out.t)
    if ot != "e4m3":
        assert np.all(np.abs(got - v) <= bound + (BF16 * (np.abs(v) + bound) if ot == "bf16" else 0.0) + 1e-38)
        return
    per = np.repeat(host(scales.t), group or d, axis=1)[:, :d]
    _, sc = oracle.quantize_e4m3(v, group)
    most = np.stack([bound[:, lo:lo + (group or d)].max(axis=1) for lo in range(0, d, group or d)], 1)
    assert np.all(np.abs(host(scales.t) - sc) <= most / 448.0 + 2 * U * sc)
    assert np.all(np.abs(got * per - v) <= np.maximum(2.0 ** -4 * np.abs(v), 2.0 ** -10 * per) * (1 + 2.0 ** -12) + 2 * bound + 8 * U * np.abs(v))


def test_add_layernorm_without_gain_and_bias_and_far_from_zero(lib):
    rng = np.random.default_rng(5)
    x = dev(rng.normal(size=(9, 264)) + 1000.0)            # a mean of a thousand deviations
    out = torch.empty(9, 264, device="cuda")
    lib.mlpmoe_add_layernorm(x, None, None, out, 9, 264, out_dtype=lib.MLPMOE_FP32, eps=1e-3, stream=stream_ptr())
    _, v = oracle.add_layernorm(host(x), None, None, None, 1e-3)
    # the mean is off by 8 + 5 + 8 + 2 roundings of 1000, and so is every z
    assert np.all(np.abs(host(out) - v) <= 25 * U * 1000 * 1.2 * (1 + np.abs(v)))


# ------------------------------------------------------------------------------------------------ the norms' gradient

GRADS = [
    # n, d, s, grad_out, grad_s, grad_x, pad
    (1, 1, "fp32", "fp32", "none", "fp32", 0), (1, 4096, "fp32", "bf16", "fp32", "fp32", 0), (3, 7, "bf16", "fp32", "none", "bf16", 1),
    (5, 8, "fp32", "fp32", "bf16", "fp32", 8), (2, 33, "fp32", "bf16", "fp32", "fp32", 0), (1001, 256, "fp32", "bf16", "fp32", "fp32", 0),
    (4100, 100, "bf16", "bf16", "bf16", "bf16", 4), (9000, 9, "fp32", "fp32", "none", "fp32", 3), (700, 257, "fp32", "bf16", "fp32", "fp32", 0),
    (1300, 896, "fp32", "bf16", "fp32", "fp32", 0), (2500, 1000, "bf16", "bf16", "bf16", "fp32", 8), (601, 1032, "fp32", "bf16", "none", "bf16", 0),
    (600, 2048, "fp32", "bf16", "fp32", "fp32", 0), (301, 2057, "bf16", "fp32", "fp32", "fp32", 3), (500, 4096, "fp32", "bf16", "fp32", "fp32", 0),
    (310, 4096, "bf16", "bf16", "bf16", "bf16", 16), (150, 4104, "fp32", "bf16", "fp32", "fp32", 0), (200, 8192, "fp32", "bf16", "bf16", "fp32", 0),
    (149, 8191, "bf16", "fp32", "none", "fp32", 0), (3, 8200, "fp32", "bf16", "fp32", "fp32", 0), (200, 20001, "bf16", "fp32", "fp32", "bf16", 0),
    (65, 32768, "fp32", "bf16", "fp32", "fp32", 0), (900, 512, "fp32", "bf16", "fp32", "fp32", 0), (333, 513, "bf16", "bf16", "fp32", "bf16", 0),
    (2400, 400, "bf16", "fp32", "bf16", "fp32", 1), (1200, 1024, "fp32", "fp32", "fp32", "fp32", 0), (700, 1025, "bf16", "bf16", "bf16", "bf16", 0),
    (300, 700, "fp32", "bf16", "fp32", "bf16", 0), (200, 1100, "bf16", "bf16", "bf16", "fp32", 4), (77, 4, "fp32", "bf16", "fp32", "bf16", 0),
    (90, 12, "bf16", "bf16", "bf16", "bf16", 4), (310, 2500, "fp32", "fp32", "bf16", "bf16", 0), (180, 4100, "fp32", "bf16", "fp32", "fp32", 0),
    (160, 5121, "bf16", "bf16", "fp32", "bf16", 0), (66, 8196, "fp32", "bf16", "fp32", "fp32", 0)]


@pytest.mark.parametrize("n,d,st,gt,rt,xt,pad", GRADS)
@pytest.mark.parametrize("layer", [False, True])
def test_norm_backward(lib, n, d, st, gt, rt, xt, pad, layer):
    rng = np.random.default_rng([d, n, 2])
    s = strided(rng.normal(size=(n, d)) * np.exp(0.5 * rng.normal(size=(n, 1))) + 0.3, st, pad)
    if n > 2:
        s[1] = 0                                           # a row of zeros: 1 / sqrt(eps)
    gv = strided(rng.normal(size=(n, d)), gt, pad)
    gs = None if rt == "none" else strided(rng.normal(size=(n, d)), rt, pad)
    gain = dev(1 + 0.2 * rng.normal(size=d)) if n != 601 else None
    want = oracle.norm_grad(layer, host(s), None if gain is None else host(gain), host(gv), None if gs is None else host(gs))
    inplace = gs is not None and rt == xt and n % 2 == 0
    gx = gs if inplace else torch.full((n, d + pad), 7.0, device="cuda").to(TORCH[xt])
    gg, gb = Guarded((d,), torch.float32), Guarded((d,), torch.float32)
    work = Guarded((lib.mlpmoe_norm_backward_workspace(n, d),), torch.uint8)
    lib.mlpmoe_norm_backward(lib.MLPMOE_LAYERNORM if layer else lib.MLPMOE_RMSNORM, s, gv, gx, n, d, work.t, work.nbytes, gain=gain, grad_s=gs,
                             grad_gain=gg.t, grad_bias=gb.t if layer else None, eps=1e-5, s_dtype=kind(lib, st), grad_out_dtype=kind(lib, gt),
                             grad_s_dtype=kind(lib, "fp32" if gs is None else rt), grad_x_dtype=kind(lib, xt), s_stride=s.stride(0),
                             grad_out_stride=gv.stride(0), grad_s_stride=0 if gs is None else gs.stride(0), grad_x_stride=gx.stride(0),
                             stream=stream_ptr())
    torch.cuda.synchronize()
    for buffer in (gg, gb, work):
        buffer.check()
    # sums over a row: up to 32 terms a thread, 5 shuffles, 32 partial sums, 70 u of the terms' sizes with the factor 1 / d.  z is off by the
    # mean's error, q by half of what the squares' mean is off by, the rest is a handful of roundings.
    z64, v64, g64 = host(s), host(gv), 1.0 if gain is None else host(gain)
    mean_abs = np.abs(z64).mean(axis=1, keepdims=True)
    off = (70 * U * mean_abs + 2 * U * np.abs(z64)) if layer else 0.0 * z64
    z = z64 - z64.mean(axis=1, keepdims=True) if layer else z64
    q = 1.0 / np.sqrt((z * z).mean(axis=1, keepdims=True) + 1e-5)
    rel = 44 * U + ((np.abs(z) * off).mean(axis=1, keepdims=True) + (off * off).mean(axis=1, keepdims=True)) * q * q * 1.01
    h = np.abs(v64 * g64)
    mh, mhz = h.mean(axis=1, keepdims=True), (h * (np.abs(z) + off)).mean(axis=1, keepdims=True)
    core = q * (h + (mh if layer else 0.0) + np.abs(z) * q * q * mhz)
    bound = core * (78 * U + 3 * rel) + q ** 3 * (off * mhz + np.abs(z) * (h * off).mean(axis=1, keepdims=True)) * 1.01
    bound = bound + 2 * U * (core + np.abs(want[0])) + 1e-37
    if xt == "bf16":
        bound = bound + BF16 * (np.abs(want[0]) + bound)
    assert np.all(np.abs(host(gx[:, :d]) - want[0]) <= bound)
    if pad and not inplace:
        assert bool((gx[:, d:] == 7.0).all())
    # over the tokens: at most n / 64 + 1 terms one after the other, then 8 rows, 37 blocks a warp and 32 warps
    terms = (n / 64 + 82) * U
    assert np.all(np.abs(host(gg.t) - want[1]) <= (np.abs(v64) * (np.abs(z) * q * (terms + rel + 3 * U) + off * q)).sum(axis=0) * 1.01 + 1e-37)
    if layer:
        assert np.all(np.abs(host(gb.t) - want[2]) <= terms * np.abs(v64).sum(axis=0) + 1e-37)


def test_norm_backward_without_sums_and_of_no_tokens(lib):
    rng = np.random.default_rng(3)
    for d in (200, 1000, 9000):
        s, gv = dev(rng.normal(size=(70, d))), dev(rng.normal(size=(70, d)), "bf16")
        gg, gb = torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
        size = lib.mlpmoe_norm_backward_workspace(70, d)
        work = torch.empty(size, dtype=torch.uint8, device="cuda")
        with_sums, alone, bias_only = (torch.empty(70, d, device="cuda") for _ in range(3))
        lib.mlpmoe_norm_backward(lib.MLPMOE_LAYERNORM, s, gv, with_sums, 70, d, work, size, grad_gain=gg, grad_bias=gb, stream=stream_ptr())
        lib.mlpmoe_norm_backward(lib.MLPMOE_LAYERNORM, s, gv, alone, 70, d, stream=stream_ptr())
        other = torch.empty(d, device="cuda")
        lib.mlpmoe_norm_backward(lib.MLPMOE_LAYERNORM, s, gv, bias_only, 70, d, work, size, grad_bias=other, stream=stream_ptr())
        assert torch.equal(with_sums, alone) and torch.equal(with_sums, bias_only) and torch.equal(gb, other)
        # no tokens: cleared
        lib.mlpmoe_norm_backward(lib.MLPMOE_LAYERNORM, None, None, None, 0, d, work, size, grad_gain=gg, grad_bias=gb, stream=stream_ptr())
        torch.cuda.synchronize()
        assert not bool(gg.any()) and not bool(gb.any())


# ------------------------------------------------------------------------------------------------ AdamW

class Param:
    """One tensor of a step: device buffers (`shift` elements off their alignment) and their values in float64."""

    def __init__(self, rng, n, pt, gt, state, copy=False, shift=0, decay=0.1):
        self.n, self.pt, self.gt, self.state, self.decay = n, pt, gt, state, decay

        def buffer(values, dtype):
            b = Guarded((n + shift,), dtype)
            b.t[shift:] = torch.from_numpy(np.asarray(values, np.float32)).cuda().to(dtype)
            return b, b.t[shift:]
        self.guards = []

        def keep(values, dtype):
            b, t = buffer(values, dtype)
            self.guards.append(b)
            return t
        self.p = keep(rng.normal(size=n) * 0.02, TORCH[pt])
        self.g = keep(rng.normal(size=n) * 1e-3, TORCH[gt])
        m, root = rng.normal(size=n) * 3e-4, np.abs(rng.normal(size=n)) * 1e-3
        root[rng.uniform(size=n) < 0.1] *= 1e-7
        self.copy = keep(np.zeros(n), torch.bfloat16) if copy else None
        if state == "fp32":
            self.m, self.v, self.ms, self.vs = keep(m, torch.float32), keep(root * root, torch.float32), None, None
        else:
            (cm, sm), (cv, sv) = oracle.adamw_blocks(m, False), oracle.adamw_blocks(root, True)
            self.m, self.v = keep(cm, TORCH["e4m3"]), keep(cv, TORCH["e4m3"])
            self.ms, self.vs = Guarded((len(sm),), torch.float32, dev(sm)), Guarded((len(sv),), torch.float32, dev(sv))
            self.guards += [self.ms, self.vs]

    def values(self):
        """(p, g, m, v)"""
        if self.state == "fp32":
            return host(self.p), host(self.g), host(self.m), host(self.v)
        per = [np.repeat(host(s.t), 128)[:self.n] for s in (self.ms, self.vs)]
        return host(self.p), host(self.g), host(self.m) * per[0], (host(self.v) * per[1]) ** 2

    def record(self, lib):
        return dict(n=self.n, param=self.p, grad=self.g, m=self.m, v=self.v, m_scale=None if self.ms is None else self.ms.t,
                    v_scale=None if self.vs is None else self.vs.t, param_bf16=self.copy, weight_decay=self.decay, param_dtype=kind(lib, self.pt),
                    grad_dtype=kind(lib, self.gt), state_dtype=kind(lib, self.state))

    def check(self, before, lr, b1, b2, eps, step, scale, noise):
        for b in self.guards:
            b.check()
        p0, g, m0, v0 = before
        decay = float(np.float32(self.decay))
        p, m, v = oracle.adamw(p0, g, m0, v0, lr, b1, b2, eps, decay, step, scale)
        # moments: the gradient's product, two products with rounded constants and a sum: 5 u of the terms' sizes (6 for the square)
        m_size, v_size = b1 * np.abs(m0) + (1 - b1) * np.abs(g * scale), b2 * v0 + (1 - b2) * (g * scale) ** 2
        m_off, v_off = 5 * U * m_size, 7 * U * v_size
        root, root_off = np.sqrt(v), 5 * U * np.sqrt(v) + TINY ** 0.5
        # the quotient: the moments' errors, root 4 u, the corrections (a logarithm, an exponential and a product) 8 u each, sum and division 4 u
        den = np.sqrt(v / (1 - b2 ** step)) + eps
        rate = lr / (1 - b1 ** step)
        p_off = 4 * U * np.abs(p0) + rate * (m_off + 28 * U * np.abs(m)) / den * 1.01 + rate * np.abs(m) / den * np.minimum(1.0, TINY ** 0.5 / den)
        got = self.values()
        if self.pt == "fp32":
            assert np.all(np.abs(got[0] - p) <= p_off + TINY)
        else:
            assert np.all(np.abs(got[0] - p) <= p_off * 1.01 + (2 if noise is not None else 1) * BF16 * np.abs(p) + TINY)
        if self.copy is not None:
            assert np.all(np.abs(host(self.copy) - p) <= p_off * 1.01 + BF16 * np.abs(p) + TINY)
        if self.state == "fp32":
            assert np.all(np.abs(got[2] - m) <= m_off + TINY) and np.all(np.abs(got[3] - v) <= v_off + TINY)
            return
        for x, x_off, codes, scales, is_root, bits in ((m, m_off, self.m, self.ms, False, noise), (root, root_off, self.v, self.vs, True, noise)):
            want, want_scale = oracle.adamw_blocks(x, is_root, noise)
            sc = host(scales.t)
            most = np.array([x_off[i:i + 128].max() for i in range(0, self.n, 128)])
            assert np.all(np.abs(sc - want_scale) <= most / 448 + 3 * U * want_scale)
            got_codes, per = host(codes), np.repeat(sc, 128)[:self.n]
            # half a step to nearest, a step with noise; a root above zero is raised to the smallest code
            steps = 2 if noise is not None else 1
            step_off = np.maximum(steps * 2.0 ** -4 * np.abs(x), (2.0 ** -9 if is_root or steps == 2 else 2.0 ** -10) * per)
            assert np.all(np.abs(got_codes * per - x) <= step_off * 1.001 + 2 * x_off)
            # and it is the oracle's code but where the value lies within its error, some 1e-5 of a step, of the border between two
            assert np.mean(got_codes != want) <= 2e-3 + 2 / self.n
            if is_root:
                assert np.all(got_codes[x > TINY ** 0.5] > 0)


SETS = [
    [(1, "fp32", "fp32", "fp32", False, 0)], [(1, "bf16", "bf16", "e4m3", False, 0)], [(127, "fp32", "bf16", "e4m3", True, 0), (129, "bf16", "fp32", "fp32", False, 0)],
    [(4096, "fp32", "bf16", "e4m3", True, 0), (4097, "fp32", "bf16", "e4m3", True, 0), (4103, "fp32", "fp32", "fp32", True, 1)],
    [(10000, "bf16", "bf16", "e4m3", False, 3), (8192, "bf16", "bf16", "fp32", False, 0), (777, "fp32", "fp32", "e4m3", True, 1)],
    [(300000, "fp32", "bf16", "e4m3", True, 0), (200001, "fp32", "fp32", "fp32", False, 0)]]


@pytest.mark.parametrize("sizes", SETS)
@pytest.mark.parametrize("stochastic", [False, True])
@pytest.mark.parametrize("step,scale", [(1, None), (1000, 0.37)])
def test_adamw(lib, sizes, stochastic, step, scale):
    rng = np.random.default_rng([step, len(sizes), sizes[0][0]])
    params = [Param(rng, n, pt, gt, state, copy, shift, decay=0.1 * (i % 2)) for i, (n, pt, gt, state, copy, shift) in enumerate(sizes)]
    before = [p.values() for p in params]
    seed = 0xABCDEF0123456789
    scale32 = 1.0 if scale is None else float(np.float32(scale))
    lib.mlpmoe_adamw(lib.mlpmoe_adamw_tensors([p.record(lib) for p in params]), 1e-3, 0.9, 0.999, 1e-8, step=step,
                     grad_scale=None if scale is None else dev([scale]), stochastic=stochastic, seed=seed, stream=stream_ptr())
    torch.cuda.synchronize()
    for i, p in enumerate(params):
        p.check(before[i], 1e-3, 0.9, 0.999, 1e-8, step, scale32, oracle.adamw_noise(seed, step, i, p.n) if stochastic else None)


def test_adamw_many_tensors_and_device_settings(lib):
    """More tensors than one launch takes, of both states mixed; step and rate from the device; the same bits as one by one."""
    rng = np.random.default_rng(9)
    kinds = [("fp32", "fp32", "fp32"), ("bf16", "bf16", "e4m3"), ("fp32", "bf16", "e4m3")]
    sizes = [int(n) for n in rng.integers(0, 400, 900)] + [9000]
    a, b = ([Param(np.random.default_rng(i), n, *kinds[i % 3], decay=0.01 * (i % 5)) if n else None for i, n in enumerate(sizes)] for _ in range(2))
    empty = dict(n=0, param=None, grad=None, m=None, v=None)
    step, lr = torch.tensor([5], device="cuda"), dev([2e-3])
    lib.mlpmoe_adamw(lib.mlpmoe_adamw_tensors([p.record(lib) if p else empty for p in a]), 0.5, 0.9, 0.99, 1e-8, step=step, lr_device=lr, stream=stream_ptr())
    for p in b:
        if p:
            lib.mlpmoe_adamw(lib.mlpmoe_adamw_tensors([p.record(lib)]), float(np.float32(2e-3)), 0.9, 0.99, 1e-8, step=5, stream=stream_ptr())
    torch.cuda.synchronize()
    for x, y in zip(a, b):
        if x:
            for name in ("p", "m", "v"):
                assert torch.equal(getattr(x, name).view(torch.uint8), getattr(y, name).view(torch.uint8)), name
            for g in x.guards:
                g.check()


@pytest.mark.parametrize("state", ["fp32", "e4m3"])
@pytest.mark.parametrize("stochastic", [False, True])
def test_adamw_gradients_that_are_not_finite_stay_alone(lib, state, stochastic):
    rng = np.random.default_rng(10)
    p, clean = (Param(np.random.default_rng(10), 700, "fp32", "fp32", state) for _ in range(2))
    at = {5: float("nan"), 200: float("inf"), 699: float("-inf")}
    clean.g[list(at)] = 0.0
    for i, value in at.items():
        p.g[i] = value
    for x in (p, clean):
        lib.mlpmoe_adamw(lib.mlpmoe_adamw_tensors([x.record(lib)]), 1e-3, stochastic=stochastic, seed=3, stream=stream_ptr())
    torch.cuda.synchronize()
    others = [i for i in range(700) if i not in at]
    for i in at:
        assert not np.isfinite(host(p.p)[i]) and not np.isfinite(host(p.m)[i]) and not np.isfinite(host(p.v)[i])
    assert np.array_equal(host(p.p)[others], host(clean.p)[others])
    for a, b in zip(p.values()[2:], clean.values()[2:]):
        assert np.all(np.isfinite(a[others]))
        if state == "fp32":
            assert np.array_equal(a[others], b[others])


def test_adamw_in_eight_bits_follows_the_moments(lib):
    """A steady gradient: with noise the stored root reaches the gradient's size (to nearest it would stay where it is)."""
    n = 128 * 400
    got = {}
    for stochastic in (False, True):
        g = torch.full((n,), 1e-3, device="cuda")
        g[::128] = 4e-3                                    # the largest of each block moves its scale
        p, m, v = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda").to(TORCH["e4m3"]), torch.zeros(n, device="cuda").to(TORCH["e4m3"])
        ms, vs = torch.zeros(n // 128, device="cuda"), torch.zeros(n // 128, device="cuda")
        tensors = lib.mlpmoe_adamw_tensors([dict(n=n, param=p, grad=g, m=m, v=v, m_scale=ms, v_scale=vs, state_dtype=lib.MLPMOE_E4M3)])
        for step in range(1, 301):
            lib.mlpmoe_adamw(tensors, 1e-5, 0.9, 0.99, 1e-8, step=step, stochastic=stochastic, seed=1, stream=stream_ptr())
            if step == 150:
                g[1::128] = 2e-3                           # twice as large from here on
        got[stochastic] = (v.float() * vs.repeat_interleave(128)).view(-1, 128)[:, 1].cpu().numpy().astype(np.float64)
    want = np.sqrt(0.99 ** 150 * (1 - 0.99 ** 150) * 1e-6 + (1 - 0.99 ** 150) * 4e-6)
    # 400 elements that wander by a few steps of 2^-3 each (deviation 6 % in the oracle's arithmetic), 1 % above on average, since
    # the square's mean is above the mean's square: within half a step of e4m3
    assert abs(got[True].mean() / want - 1) < 2.0 ** -4
    assert np.all(np.abs(got[False] / want - 1) < 1.0)


# ------------------------------------------------------------------------------------------------ together

def training_step(lib, seed=0, n=200, d=136, B=6, k=2, inter=48, align=16):
    """norm -> router -> sorted rows -> the branches' products -> sum, and back to every gradient: device results and float64 ones."""
    gen = torch.Generator().manual_seed(seed)

    def normal(*shape, std=1.0):
        return torch.randn(*shape, generator=gen, dtype=torch.float64).mul(std).float().double()
    x, gain, Wr = normal(n, d), 1 + normal(d, std=0.1), normal(d, B, std=0.1)
    Wg, Wu, Wd = normal(B, d, inter, std=0.1), normal(B, d, inter, std=0.1), normal(B, inter, d, std=0.1)
    dy = normal(n, d)
    c = {name: t.float().cuda() for name, t in dict(x=x, gain=gain, Wr=Wr, Wg=Wg, Wu=Wu, Wd=Wd, dy=dy).items()}
    f32 = dict(rows_dtype=lib.MLPMOE_FP32)
    st = stream_ptr()
    e = lambda *shape, dtype=torch.float32: torch.empty(*shape, dtype=dtype, device="cuda")  # noqa: E731
    i32 = torch.int32
    s, v = e(n, d), e(n, d)
    lib.mlpmoe_add_rmsnorm(c["x"], None, s, v, n, d, gain=c["gain"], out_dtype=lib.MLPMOE_FP32, stream=st)
    logits = v @ c["Wr"]
    select, route_counts, prob, loss = e(n, B, dtype=torch.uint8), e(B + 1, dtype=i32), e(B), e(1)
    size = lib.mlpmoe_route_workspace(n, B)
    lib.mlpmoe_route(logits, n, B, k, select, route_counts, prob, loss, e(size, dtype=torch.uint8), size, stream=st)
    R = lib.mlpmoe_sort_rows(n, B, k, align)
    offsets, counts, row_token, token_row, token_branch = e(B + 1, dtype=i32), e(B, dtype=i32), e(R, dtype=i32), e(n, k, dtype=i32), e(n, k, dtype=i32)
    size = lib.mlpmoe_sort_workspace(n, B)
    lib.mlpmoe_sort_tokens(select, n, B, k, offsets, counts, row_token, R, token_row, e(size, dtype=torch.uint8), size, align=align,
                           token_branch=token_branch, stream=st)
    rows = torch.zeros(R, d, device="cuda")
    lib.mlpmoe_dispatch(v, rows, n, d, B, k, offsets, counts, token_row, R, align=align, dtype=lib.MLPMOE_FP32, stream=st)
    chosen = logits.gather(1, token_branch.long())
    weight = torch.softmax(chosen, 1)
    at = offsets.tolist()
    out, saved = torch.zeros(R, d, device="cuda"), []
    for b in range(B):
        r = rows[at[b]:at[b + 1]]
        g, u = r @ c["Wg"][b], r @ c["Wu"][b]
        h = torch.nn.functional.silu(g) * u
        out[at[b]:at[b + 1]] = h @ c["Wd"][b]
        saved.append((r, g, u, h))
    y = e(n, d)
    lib.mlpmoe_combine(out, R, token_row, k, y, n, d, weight=weight, residual=s, stream=st, **f32)
    # back
    d_out, d_weight = torch.zeros(R, d, device="cuda"), e(n, k)
    lib.mlpmoe_combine_backward(c["dy"], out, R, token_row, k, d_out, d_weight, n, d, weight=weight, B=B, align=align, offsets=offsets, counts=counts,
                                stream=st, **f32)
    d_rows, grads = torch.zeros(R, d, device="cuda"), {"Wg": [], "Wu": [], "Wd": []}
    for b in range(B):
        r, g, u, h = saved[b]
        do = d_out[at[b]:at[b + 1]]
        dh = do @ c["Wd"][b].t()
        sig = torch.sigmoid(g)
        dg, du = dh * u * sig * (1 + g * (1 - sig)), dh * g * sig
        d_rows[at[b]:at[b + 1]] = dg @ c["Wg"][b].t() + du @ c["Wu"][b].t()
        grads["Wg"].append(r.t() @ dg), grads["Wu"].append(r.t() @ du), grads["Wd"].append(h.t() @ do)
    grads = {name: torch.stack(g) for name, g in grads.items()}
    d_logits = e(n, B)
    lib.mlpmoe_route_backward(logits, route_counts, d_logits, n, B, stream=st)
    d_logits.scatter_add_(1, token_branch.long(), weight * (d_weight - (weight * d_weight).sum(1, keepdim=True)))
    grads["Wr"] = v.t() @ d_logits
    d_v = e(n, d)
    via_logits = d_logits @ c["Wr"].t()
    lib.mlpmoe_combine(d_rows, R, token_row, k, d_v, n, d, residual=via_logits, stream=st, **f32)      # the gradient of the dispatch
    size = lib.mlpmoe_norm_backward_workspace(n, d)
    grads["x"], grads["gain"] = e(n, d), e(d)
    lib.mlpmoe_norm_backward(lib.MLPMOE_RMSNORM, s, d_v, grads["x"], n, d, e(size, dtype=torch.uint8), size, gain=c["gain"], grad_s=c["dy"],
                             grad_gain=grads["gain"], grad_out_dtype=lib.MLPMOE_FP32, stream=st)
    torch.cuda.synchronize()
    # the same in float64 by automatic differentiation, for the selection that was made
    leaves = {name: t.clone().requires_grad_() for name, t in dict(x=x, gain=gain, Wr=Wr, Wg=Wg, Wu=Wu, Wd=Wd).items()}
    v64 = leaves["x"] / torch.sqrt((leaves["x"] ** 2).mean(1, keepdim=True) + 1e-6) * leaves["gain"]
    l64 = v64 @ leaves["Wr"]
    mask = select.cpu().bool()
    w64 = torch.softmax(l64.masked_fill(~mask, float("-inf")), 1)
    y64 = leaves["x"]
    for b in range(B):
        y64 = y64 + w64[:, b:b + 1] * ((torch.nn.functional.silu(v64 @ leaves["Wg"][b]) * (v64 @ leaves["Wu"][b])) @ leaves["Wd"][b])
    f = mask.sum(0).double() / mask.sum()
    total = (y64 * dy).sum() + B * (f * torch.softmax(l64, 1).mean(0)).sum()
    total.backward()
    return c, y, grads, y64.detach(), {name: t.grad for name, t in leaves.items()}


def test_a_training_step_around_a_routed_layer(lib):
    old = torch.backends.cuda.matmul.allow_tf32
    torch.backends.cuda.matmul.allow_tf32 = False
    try:
        c, y, grads, want_y, want = training_step(lib)
    finally:
        torch.backends.cuda.matmul.allow_tf32 = old
    # fp32 throughout: sums of at most 200 terms in each of about 8 stages, in terms of the largest value
    assert float((y.cpu().double() - want_y).abs().max() / want_y.abs().max()) <= 8 * 200 * U
    for name, g in grads.items():
        assert float((g.cpu().double() - want[name]).abs().max() / want[name].abs().max()) <= 8 * 200 * U, name
    # and the step itself, on all weights at once
    names = ["Wr", "gain", "Wg", "Wu", "Wd"]
    state = {name: (torch.zeros_like(c[name]), torch.zeros_like(c[name])) for name in names}
    before = {name: c[name].cpu().double() for name in names}
    tensors = lib.mlpmoe_adamw_tensors([dict(n=c[name].numel(), param=c[name], grad=grads[name].contiguous(), m=state[name][0], v=state[name][1],
                                             weight_decay=0.0 if name == "gain" else 0.1) for name in names])
    lib.mlpmoe_adamw(tensors, 1e-2, step=1, stream=stream_ptr())
    torch.cuda.synchronize()
    for name in names:
        g = grads[name].cpu().double()
        p, m, v = oracle.adamw(before[name].numpy(), g.numpy(), 0.0, 0.0, 1e-2, 0.9, 0.999, 1e-8, 0.0 if name == "gain" else float(np.float32(0.1)), 1)
        assert np.all(np.abs(host(c[name]) - p) <= 4 * U * np.abs(before[name].numpy()) + 1e-2 * 64 * U)      # the quotient is 1 at the first step
        assert np.all(np.abs(host(state[name][0]) - m) <= 5 * U * np.abs(m) + TINY)


def test_captured_on_another_stream_and_replayed(lib):
    """The calls of a step in a graph, captured on a side stream: replays follow new inputs, and the workspaces are the graph's own."""
    n, B, k, d, align = 700, 12, 3, 520, 8
    rng = np.random.default_rng(21)
    plan = Plan(lib, selection(rng, n, B, 3), k, align)
    x, w = dev(rng.normal(size=(n, d))), dev(rng.normal(size=(n, k)))
    rows, y, grad_w = torch.zeros(plan.rows, d, device="cuda"), torch.zeros(n, d, device="cuda"), torch.zeros(n, k, device="cuda")
    gx, gg, gb = torch.zeros(n, d, device="cuda"), torch.zeros(d, device="cuda"), torch.zeros(d, device="cuda")
    size = lib.mlpmoe_norm_backward_workspace(n, d)
    work = torch.empty(size, dtype=torch.uint8, device="cuda")
    p, m, v, step = (torch.zeros(d, device="cuda") for _ in range(3)), None, None, torch.tensor([0], device="cuda")
    p, m, v = p
    tensors = lib.mlpmoe_adamw_tensors([dict(n=d, param=p, grad=gg, m=m, v=v)])

    def calls(stream):
        plan.run(lib, stream)
        lib.mlpmoe_dispatch(x, rows, n, d, B, k, plan.offsets.t, plan.counts.t, plan.token_row.t, plan.rows, align=align, dtype=lib.MLPMOE_FP32, stream=stream)
        lib.mlpmoe_combine(rows, plan.rows, plan.token_row.t, k, y, n, d, weight=w, residual=x, rows_dtype=lib.MLPMOE_FP32, stream=stream)
        lib.mlpmoe_combine_backward(y, rows, plan.rows, plan.token_row.t, k, rows, grad_w, n, d, weight=w, B=B, align=align, offsets=plan.offsets.t,
                                    counts=plan.counts.t, rows_dtype=lib.MLPMOE_FP32, stream=stream)
        lib.mlpmoe_norm_backward(lib.MLPMOE_LAYERNORM, x, y, gx, n, d, work, size, grad_gain=gg, grad_bias=gb, grad_out_dtype=lib.MLPMOE_FP32, stream=stream)
        step.add_(1)
        lib.mlpmoe_adamw(tensors, 1e-2, step=step, stream=stream)
    results = [rows, y, grad_w, gx, gg, gb, p, m, v]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls(side.cuda_stream)                            # eager on the side stream
    torch.cuda.synchronize()
    plan.check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        calls(torch.cuda.current_stream().cuda_stream)
    for i in range(3):
        select = selection(rng, n, B, 2 + i)
        plan.want = oracle.sort_tokens(select, k, align)
        plan.used = len(plan.want["row_token"])
        plan.row_token.t.view(torch.uint8).fill_(POISON)
        plan.select.copy_(torch.from_numpy(select.reshape(-1)))
        x.copy_(dev(rng.normal(size=(n, d))))
        rows.zero_()
        start = [t.clone() for t in (p, m, v)]
        graph.replay()
        torch.cuda.synchronize()
        plan.check()
        replayed = [t.clone() for t in results]
        for t, s in zip((p, m, v), start):
            t.copy_(s)
        rows.zero_()
        step.sub_(1)
        calls(stream_ptr())
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(replayed, results))
        assert int(step) == i + 2
    graph.reset()


def test_rows_and_elements_past_32_bit_offsets(lib):
    """Rows whose elements lie past 2^31 and 2^32 bytes, and a tensor with more than 2^31 elements."""
    d, R = 32768, 70000
    rows = torch.empty(R, d, dtype=torch.bfloat16, device="cuda")
    far = [0, 40000, 65535, 65536, R - 1]
    place = ints([[r] for r in far])
    x = dev(np.random.default_rng(1).normal(size=(len(far), d)), "bf16")
    lib.mlpmoe_dispatch(x, rows, len(far), d, 1, 1, None, None, place, R, stream=stream_ptr())
    assert torch.equal(rows[far], x)
    y = torch.empty(len(far), d, dtype=torch.bfloat16, device="cuda")
    lib.mlpmoe_combine(rows, R, place, 1, y, len(far), d, y_dtype=lib.MLPMOE_BF16, stream=stream_ptr())
    assert torch.equal(y, x)
    gw = torch.empty(len(far), 1, device="cuda")
    lib.mlpmoe_combine_backward(x, rows, R, place, 1, rows, gw, len(far), d, weight=torch.full((len(far), 1), 2.0, device="cuda"),
                                grad_y_dtype=lib.MLPMOE_BF16, stream=stream_ptr())
    assert torch.equal(rows[far].float(), 2 * x.float())
    del rows
    n = (1 << 31) + 1000
    p, g = torch.zeros(n, dtype=torch.bfloat16, device="cuda"), torch.full((n,), 1e-3, dtype=torch.bfloat16, device="cuda")
    m, v = (torch.zeros(n, dtype=torch.uint8, device="cuda").view(TORCH["e4m3"]) for _ in range(2))
    ms, vs = (torch.zeros(-(-n // 128), device="cuda") for _ in range(2))
    tensors = lib.mlpmoe_adamw_tensors([dict(n=n, param=p, grad=g, m=m, v=v, m_scale=ms, v_scale=vs, param_dtype=lib.MLPMOE_BF16,
                                             grad_dtype=lib.MLPMOE_BF16, state_dtype=lib.MLPMOE_E4M3)])
    lib.mlpmoe_adamw(tensors, 0.5, step=1, stream=stream_ptr())
    torch.cuda.synchronize()
    # every element steps by lr, 0.5, within bf16's rounding (the same gradient everywhere)
    lo, hi = p.aminmax()
    assert float(lo) == float(hi) == -0.5
    assert bool((m.view(torch.uint8) == 0x7E).all()) and bool((v.view(torch.uint8) == 0x7E).all())      # 448: each is its block's largest


def test_adamw_past_32_bit_elements(lib):
    """Elements on both sides of 2^32, with noise: their codes, scales and params are the oracle's."""
    n = (1 << 32) + 4096
    if torch.cuda.mem_get_info()[0] < 6 * n + (4 << 30):
        pytest.skip("not enough free memory")
    p, g = (torch.zeros(n, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    m, v = (torch.zeros(n, dtype=torch.uint8, device="cuda").view(TORCH["e4m3"]) for _ in range(2))
    ms, vs = (torch.zeros(n // 128, device="cuda") for _ in range(2))
    rng = np.random.default_rng(2)
    parts = {first: (dev(rng.normal(size=2048) * 0.02, "bf16"), dev(rng.normal(size=2048) * 1e-3, "bf16")) for first in (0, (1 << 32) - 2048, 1 << 32, n - 2048)}
    for first, (pp, gg) in parts.items():
        p[first:first + 2048], g[first:first + 2048] = pp, gg
    tensors = lib.mlpmoe_adamw_tensors([dict(n=n, param=p, grad=g, m=m, v=v, m_scale=ms, v_scale=vs, param_dtype=lib.MLPMOE_BF16,
                                             grad_dtype=lib.MLPMOE_BF16, state_dtype=lib.MLPMOE_E4M3)])
    lib.mlpmoe_adamw(tensors, 1e-3, step=3, stochastic=True, seed=77, stream=stream_ptr())
    torch.cuda.synchronize()
    for first, (pp, gg) in parts.items():
        want_p, want_m, want_v = oracle.adamw(host(pp), host(gg), 0.0, 0.0, 1e-3, 0.9, 0.999, 1e-8, 0.0, 3)
        noise = oracle.adamw_noise(77, 3, 0, 2048, first)
        at = slice(first, first + 2048)
        for x, codes, is_root in ((want_m, m, False), (np.sqrt(want_v), v, True)):
            assert np.mean(host(codes[at]) != oracle.adamw_blocks(x, is_root, noise)[0]) <= 2e-3
        assert np.all(np.abs(host(p[at]) - want_p) <= 2 * BF16 * np.abs(want_p) + 1e-3 * 64 * U)
    assert not bool(p[2048:1 << 20].any()) and not bool(m.view(torch.uint8)[2048:1 << 20].any())      # zeros stay zeros


# ------------------------------------------------------------------------------------------------ the same bits, and several threads

def test_the_same_bits_every_time(lib):
    rng = np.random.default_rng(31)
    plan = Plan(lib, selection(rng, 3000, 40, 5), 5, 16)
    gy, rows, w = dev(rng.normal(size=(3000, 264))), dev(rng.normal(size=(plan.rows, 264)), "bf16"), dev(rng.normal(size=(3000, 5)))
    s, gv = dev(rng.normal(size=(3000, 264))), dev(rng.normal(size=(3000, 264)), "bf16")
    size = lib.mlpmoe_norm_backward_workspace(3000, 264)
    work = torch.empty(size, dtype=torch.uint8, device="cuda")

    def once():
        out = [torch.zeros(3000, 264, device="cuda"), torch.zeros_like(rows), torch.zeros(3000, 5, device="cuda"), torch.zeros(3000, 264, device="cuda"),
               torch.zeros(264, device="cuda"), torch.zeros(264, device="cuda")]
        plan.run(lib)
        lib.mlpmoe_combine(rows, plan.rows, plan.token_row.t, 5, out[0], 3000, 264, weight=w, residual=gy, stream=stream_ptr())
        lib.mlpmoe_combine_backward(gy, rows, plan.rows, plan.token_row.t, 5, out[1], out[2], 3000, 264, weight=w, B=40, align=16,
                                    offsets=plan.offsets.t, counts=plan.counts.t, stream=stream_ptr())
        lib.mlpmoe_norm_backward(lib.MLPMOE_LAYERNORM, s, gv, out[3], 3000, 264, work, size, grad_s=gy, grad_gain=out[4], grad_bias=out[5], stream=stream_ptr())
        return out
    first = once()
    for _ in range(3):
        work.fill_(0xEE)
        assert all(torch.equal(a, b) for a, b in zip(first, once()))


def test_calls_from_two_threads(lib):
    """Two host threads with sizes and types of their own, on streams of their own, as often as one thread after the other."""
    import threading
    jobs = []
    for seed, (n, d, st, gt) in enumerate([(300, 4096, "fp32", "fp32"), (500, 520, "bf16", "bf16")]):
        rng = np.random.default_rng(seed)
        s, gv, gs = dev(rng.normal(size=(n, d)), st), dev(rng.normal(size=(n, d)), gt), dev(rng.normal(size=(n, d)))
        size = lib.mlpmoe_norm_backward_workspace(n, d)
        out = [torch.zeros(n, d, device="cuda"), torch.zeros(d, device="cuda"), torch.zeros(n, d, device="cuda")]
        jobs.append((n, d, st, gt, s, gv, gs, size, torch.empty(size, dtype=torch.uint8, device="cuda"), out))

    def run(job, stream):
        n, d, st, gt, s, gv, gs, size, work, out = job
        for _ in range(50):
            lib.mlpmoe_norm_backward(lib.MLPMOE_RMSNORM, s, gv, out[0], n, d, work, size, grad_s=gs, grad_gain=out[1], s_dtype=kind(lib, st),
                                     grad_out_dtype=kind(lib, gt), stream=stream)
            lib.mlpmoe_add_layernorm(s, gs, None, out[2], n, d, x_dtype=kind(lib, st), out_dtype=lib.MLPMOE_FP32, stream=stream)
    wants = []
    for job in jobs:
        run(job, stream_ptr())
        torch.cuda.synchronize()
        wants.append([t.clone() for t in job[-1]])
        for t in job[-1]:
            t.zero_()
    torch.cuda.synchronize()
    streams, errors = [torch.cuda.Stream() for _ in jobs], []

    def guarded(job, stream):
        try:
            run(job, stream.cuda_stream)
        except Exception as e:      # noqa: BLE001 - a thread's failure is the test's
            errors.append(e)
    threads = [threading.Thread(target=guarded, args=(job, stream)) for job, stream in zip(jobs, streams)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors
    for job, want in zip(jobs, wants):
        assert all(torch.equal(a, b) for a, b in zip(job[-1], want))
