"""GPU tests of the operators of a training step, beside tests/test_gpu_training.py: rounding with noise and to nearest, scales, far offsets, very
large batches."""
import numpy as np
import pytest
import torch

import oracle
from tests.helpers import Guarded, stream_ptr
from tests.test_gpu_operators import TORCH, U, dev, host
from tests.test_gpu_training import TINY, Param, Plan, selection

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------ params in bf16 with noise

def step_of(before, lr, b1, b2, eps, decay, step, scale):
    """(the params after a step, how far fp32 may be off them): the moments' errors and 28 roundings of the quotient, 4 of the param."""
    p0, g, m0, v0 = before
    p, m, v = oracle.adamw(p0, g, m0, v0, lr, b1, b2, eps, decay, step, scale)
    m_off = 5 * U * (b1 * np.abs(m0) + (1 - b1) * np.abs(g * scale))
    den, rate = np.sqrt(v / (1 - b2 ** step)) + eps, lr / (1 - b1 ** step)
    return p, 4 * U * np.abs(p0) + rate * (m_off + 28 * U * np.abs(m)) / den * 1.01 + rate * np.abs(m) / den * np.minimum(1.0, TINY ** 0.5 / den)


def check_rounded_with_noise(got, p, p_off, noise):
    """The oracle's neighbour but where the fp32 value and the oracle's lie on two sides of the noise's border: the border is at one of
    2^16 places a step, so the odds are the distance over 2^16 units of the last place (half of one for the oracle's own rounding)."""
    want = oracle.bf16_up_or_down(p, noise)
    unit = 2.0 ** (np.floor(np.log2(np.abs(p))) - 23)
    odds = np.minimum(1.0, (p_off / unit + 0.5) * 2.0 ** -16).sum()
    wrong = got != want
    assert wrong.sum() <= odds + 5 * np.sqrt(odds) + 5, (int(wrong.sum()), odds)
    step = unit * 65536
    assert np.all(np.abs(got - p) <= step * (1 + 2.0 ** -16) + 2 * p_off)
    # no drift: a coin of deviation half a step at most, and the fp32 value's own error
    drift = np.mean((np.abs(got) - np.abs(p)) / step)
    assert abs(drift) <= 5 * 0.5 / np.sqrt(p.size) + np.mean(p_off / step), drift


@pytest.mark.parametrize("n,gt,state,shift", [(200003, "bf16", "e4m3", 0), (150000, "fp32", "fp32", 0), (70001, "fp32", "e4m3", 3), (50000, "bf16", "fp32", 1)])
@pytest.mark.parametrize("step,scale", [(1, 1.0), (1000, 0.37)])
def test_bf16_params_rounded_with_noise(lib, n, gt, state, shift, step, scale):
    rng = np.random.default_rng([n, step])
    params = [Param(rng, n, "bf16", gt, state, shift=shift, decay=0.1), Param(rng, 3000, "bf16", gt, state, shift=shift, decay=0.0)]
    before = [p.values() for p in params]
    seed = 0x0123456789ABCDEF + step
    scale32 = float(np.float32(scale))
    lib.mlpmoe_adamw(lib.mlpmoe_adamw_tensors([p.record(lib) for p in params]), 1e-3, 0.9, 0.999, 1e-8, step=step, grad_scale=dev([scale]),
                     stochastic=True, seed=seed, stream=stream_ptr())
    torch.cuda.synchronize()
    for i, param in enumerate(params):
        p, p_off = step_of(before[i], 1e-3, 0.9, 0.999, 1e-8, float(np.float32(param.decay)), step, scale32)
        check_rounded_with_noise(host(param.p), p, p_off, oracle.adamw_noise(seed, step, i, param.n))
        for b in param.guards:
            b.check()


FAR = 1 << 32


def far_step(lib):
    """A step over more than 2^32 elements with noise, zeros but for four stretches: {first: (p, g)} and the buffers after it."""
    n = FAR + 4096
    if torch.cuda.mem_get_info()[0] < 6 * n + (4 << 30):
        pytest.skip("not enough free memory")
    p, g = (torch.zeros(n, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    m, v = (torch.zeros(n, dtype=torch.uint8, device="cuda").view(TORCH["e4m3"]) for _ in range(2))
    ms, vs = (torch.zeros(n // 128, device="cuda") for _ in range(2))
    rng = np.random.default_rng(12)
    parts = {first: (dev(rng.normal(size=2048) * 0.02, "bf16"), dev(rng.normal(size=2048) * 1e-3, "bf16")) for first in (0, FAR - 2048, FAR, n - 2048)}
    for first, (pp, gg) in parts.items():
        p[first:first + 2048], g[first:first + 2048] = pp, gg
    tensors = lib.mlpmoe_adamw_tensors([dict(n=n, param=p, grad=g, m=m, v=v, m_scale=ms, v_scale=vs, param_dtype=lib.MLPMOE_BF16,
                                             grad_dtype=lib.MLPMOE_BF16, state_dtype=lib.MLPMOE_E4M3)])
    lib.mlpmoe_adamw(tensors, 1e-3, step=3, stochastic=True, seed=78, stream=stream_ptr())
    torch.cuda.synchronize()
    return {first: (host(pp), host(gg)) for first, (pp, gg) in parts.items()}, p, ms, vs


def test_bf16_params_past_32_bit_elements_rounded_with_noise(lib):
    parts, p, _, _ = far_step(lib)
    for first, (p0, g) in parts.items():
        zero = np.zeros(2048)
        want, off = step_of((p0, g, zero, zero), 1e-3, 0.9, 0.999, 1e-8, 0.0, 3, 1.0)
        check_rounded_with_noise(host(p[first:first + 2048]), want, off, oracle.adamw_noise(78, 3, 0, 2048, first))


# ------------------------------------------------------------------------------------------------ 8-bit moments: scales, and to nearest

def test_scales_past_32_bit_elements(lib):
    """The scales of the stretches on both sides of 2^32, and those of zeros everywhere else."""
    parts, _, ms, vs = far_step(lib)
    rest = torch.ones(ms.numel(), dtype=torch.bool, device="cuda")
    for first, (_, g) in parts.items():
        at = slice(first // 128, first // 128 + 16)
        rest[at] = False
        m, root = 0.1 * g, np.sqrt(0.001) * np.abs(g)
        for x, scales, off in ((m, ms, 5 * U), (root, vs, 5 * U)):
            want = oracle.adamw_blocks(x, False)[1]
            # the largest value's error, then the quotient by 448: 3 u
            assert np.all(np.abs(host(scales[at]) - want) <= (off + 3 * U) * want)
    for scales in (ms, vs):
        assert bool((scales[rest] == 2.0 ** -126).all())


def test_roots_to_nearest_stay_behind(lib):
    """The arithmetic of 300 steps to nearest in 64 bits, block by block, and that it does stay behind what the gradients ask for."""
    n, lr, b1, b2, eps = 128 * 400, 1e-5, 0.9, 0.99, 1e-8
    g = np.full(128, float(np.float32(1e-3)))
    g[0] = float(np.float32(4e-3))
    p, m, v = np.zeros(128), np.zeros(128), np.zeros(128)
    gd = dev(np.tile(g, n // 128))
    pd, md, vd = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda").to(TORCH["e4m3"]), torch.zeros(n, device="cuda").to(TORCH["e4m3"])
    ms, vs = torch.zeros(n // 128, device="cuda"), torch.zeros(n // 128, device="cuda")
    tensors = lib.mlpmoe_adamw_tensors([dict(n=n, param=pd, grad=gd, m=md, v=vd, m_scale=ms, v_scale=vs, state_dtype=lib.MLPMOE_E4M3)])
    for step in range(1, 301):
        lib.mlpmoe_adamw(tensors, lr, b1, b2, eps, step=step, stream=stream_ptr())
        p, m, v = oracle.adamw(p, g, m, v, lr, b1, b2, eps, 0.0, step)
        (cm, sm), (cv, sv) = oracle.adamw_blocks(m, False), oracle.adamw_blocks(np.sqrt(v), True)
        m, v = cm * sm[0], (cv * sv[0]) ** 2
        if step == 150:
            g[1] = float(np.float32(2e-3))
            gd[1::128] = 2e-3
    got = host((vd.float() * vs.repeat_interleave(128)).view(-1, 128))
    assert np.all(got == got[0])                           # every block has the same values, and the rounding no noise
    assert np.all(np.abs(got[0] - np.sqrt(v)) <= 2.0 ** -3 * np.sqrt(v))      # one step of e4m3, where a value lies at a border
    want = np.sqrt(0.99 ** 150 * (1 - 0.99 ** 150) * 1e-6 + (1 - 0.99 ** 150) * 4e-6)
    assert got[0, 1] < 0.75 * want


# ------------------------------------------------------------------------------------------------ rows past 32-bit offsets

def test_weights_gradient_of_rows_past_32_bit_offsets(lib):
    d, R = 32768, 70000
    far = [0, 40000, 65535, 65536, R - 1]
    rng = np.random.default_rng(3)
    x, gy = dev(rng.normal(size=(len(far), d)), "bf16"), dev(rng.normal(size=(len(far), d)), "bf16")
    rows = torch.full((R, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    rows[far] = x
    place = torch.tensor([[r] for r in far], dtype=torch.int32, device="cuda")
    gw, alone = torch.empty(len(far), 1, device="cuda"), torch.empty(len(far), 1, device="cuda")
    lib.mlpmoe_combine_backward(gy, rows, R, place, 1, None, alone, len(far), d, grad_y_dtype=lib.MLPMOE_BF16, stream=stream_ptr())
    lib.mlpmoe_combine_backward(gy, rows, R, place, 1, rows, gw, len(far), d, grad_y_dtype=lib.MLPMOE_BF16, stream=stream_ptr())
    torch.cuda.synchronize()
    terms = host(gy) * host(x)
    # a thread's 32 terms, five steps in a warp, 32 warps one after the other: fewer than 80 roundings of partial sums
    for got in (alone, gw):
        assert np.all(np.abs(host(got)[:, 0] - terms.sum(1)) <= 80 * U * np.abs(terms).sum(1))
    assert torch.equal(rows[far], gy)


# ------------------------------------------------------------------------------------------------ the order of very large batches

@pytest.mark.parametrize("n,B,slots,align,mean", [
    (606208, 32, 2, 128, 1), (606209, 32, 2, 128, 1), (303105, 256, 1, 1, 2), (320001, 256, 2, 16, 2), (620001, 3, 2, 1, 1), (483000, 100, 3, 64, 2),
    (2500001, 17, 1, 1, 1)])
def test_sort_tokens_of_more_tiles_than_are_aimed_at(lib, monkeypatch, n, B, slots, align, mean):
    """From 592 tiles of the largest size on, more tiles are made; and the workspace of a larger batch serves."""
    monkeypatch.setattr(oracle, "sort_tokens", oracle.sort_tokens_of_many)
    plan = Plan(lib, selection(np.random.default_rng([n, B]), n, B, mean), slots, align)
    plan.check()
    plan.work = Guarded((lib.mlpmoe_sort_workspace(3 * n, B),), torch.uint8)
    plan.work.t.fill_(0xEE)
    for buffer in (plan.offsets, plan.counts, plan.token_row, plan.token_branch):
        buffer.t.fill_(-7)
    plan.run(lib)
    plan.check()


# ------------------------------------------------------------------------------------------------ calls again

def test_a_step_with_gradients_that_move(lib):
    """A list whose gradients' addresses alone are renewed, against one built anew for every step."""
    kinds = [(5000, "fp32", "bf16", "e4m3"), (777, "bf16", "fp32", "fp32"), (4096, "fp32", "fp32", "fp32")]
    a, b = ([Param(np.random.default_rng(i), *k) for i, k in enumerate(kinds)] for _ in range(2))
    tensors = lib.mlpmoe_adamw_tensors([dict(p.record(lib), grad=p.g.data_ptr()) for p in a])
    rng = np.random.default_rng(5)
    kept = []
    for step in (1, 2, 3):
        grads = [dev(rng.normal(size=n) * 1e-3, gt) for n, _, gt, _ in kinds]
        kept.append(grads)                                 # the next step's lie elsewhere
        for t, g in zip(tensors, grads):
            t.grad = g.data_ptr()
        lib.mlpmoe_adamw(tensors, 1e-3, step=step, stochastic=True, seed=4, stream=stream_ptr())
        anew = lib.mlpmoe_adamw_tensors([dict(p.record(lib), grad=g) for p, g in zip(b, grads)])
        lib.mlpmoe_adamw(anew, 1e-3, step=step, stochastic=True, seed=4, stream=stream_ptr())
        torch.cuda.synchronize()
        for x, y in zip(a, b):
            for name in ("p", "m", "v"):
                assert torch.equal(getattr(x, name).view(torch.uint8), getattr(y, name).view(torch.uint8)), (step, name)


@pytest.mark.parametrize("pt,gt,state,copy,shift", [("fp32", "bf16", "e4m3", True, 0), ("bf16", "bf16", "e4m3", False, 0), ("bf16", "fp32", "fp32", False, 1)])
def test_a_step_gives_the_same_bits_every_time(lib, pt, gt, state, copy, shift):
    """Also while steps over other tensors are under way on another stream."""
    params = Param(np.random.default_rng(8), 1 << 20, pt, gt, state, copy, shift)
    other = Param(np.random.default_rng(9), 1 << 22, "fp32", "bf16", "e4m3")
    start = [b.raw.clone() for b in params.guards]
    one, two = (lib.mlpmoe_adamw_tensors([p.record(lib)]) for p in (params, other))
    side = torch.cuda.Stream()
    wants = None
    for again in range(5):
        for b, s in zip(params.guards, start):
            b.raw.copy_(s)
        torch.cuda.synchronize()
        for _ in range(again):
            lib.mlpmoe_adamw(two, 1e-3, step=1, stochastic=True, seed=2, stream=side.cuda_stream)
        for step in (1, 2):
            lib.mlpmoe_adamw(one, 1e-3, step=step, stochastic=True, seed=2, stream=stream_ptr())
        torch.cuda.synchronize()
        got = [b.raw.clone() for b in params.guards]
        wants = wants or got
        assert all(torch.equal(x, y) for x, y in zip(got, wants))
    assert any(not torch.equal(x, y) for x, y in zip(start, wants))


# ------------------------------------------------------------------------------------------------ 8-bit moments bit by bit

@pytest.mark.parametrize("n,pt,gt,shift", [(200003, "fp32", "bf16", 0), (128 * 1000, "bf16", "bf16", 0), (70001, "fp32", "fp32", 3), (50, "bf16", "fp32", 1)])
@pytest.mark.parametrize("noisy,scale", [(False, None), (True, 0.5), (True, 0.37)])
def test_codes_and_scales_bit_by_bit(lib, n, pt, gt, shift, noisy, scale):
    """Three steps in a row: a code that were another one would move the next step's scale."""
    rng = np.random.default_rng([n, 3])
    param = Param(rng, n, pt, gt, "e4m3", shift=shift)
    tensors = lib.mlpmoe_adamw_tensors([param.record(lib)])
    state = [host(t) for t in (param.m, param.ms.t, param.v, param.vs.t)]
    for step in (1, 2, 3):
        param.g.copy_(dev(rng.normal(size=n) * 1e-3))
        lib.mlpmoe_adamw(tensors, 1e-3, 0.9, 0.999, 1e-8, step=step, grad_scale=None if scale is None else dev([scale]), stochastic=noisy, seed=21,
                         stream=stream_ptr())
        torch.cuda.synchronize()
        m, ms, v, vs = state
        state = oracle.adamw_moments_fp32(host(param.g), m, ms, v, vs, 0.9, 0.999, 1.0 if scale is None else scale,
                                          oracle.adamw_noise(21, step, 0, n) if noisy else None)
        for name, got, want in zip(("m", "m_scale", "v", "v_scale"), (param.m, param.ms.t, param.v, param.vs.t), state):
            assert np.array_equal(host(got), want), (step, name, int((host(got) != want).sum()))


@pytest.mark.parametrize("noisy", [False, True])
def test_codes_and_scales_bit_by_bit_of_every_size(lib, noisy):
    """Gradients from 2^-80 to 2^55, with zeros, blocks of one size and blocks of many: squares below fp32's normal range among them."""
    rng = np.random.default_rng(30)
    n = 128 * 3000
    size = np.where(np.arange(n) // 128 % 2 == 0, np.repeat(rng.uniform(-80, 55, n // 128), 128), rng.uniform(-80, 55, n))
    param = Param(rng, n, "fp32", "fp32", "e4m3")
    for t in (param.m, param.v, param.ms.t, param.vs.t):
        t.zero_()
    tensors = lib.mlpmoe_adamw_tensors([param.record(lib)])
    state = [host(t) for t in (param.m, param.ms.t, param.v, param.vs.t)]
    for step in (1, 2, 3):
        g = rng.normal(size=n) * 2.0 ** size * (rng.uniform(size=n) < 0.9)
        param.g.copy_(dev(g))
        lib.mlpmoe_adamw(tensors, 1e-3, 0.9, 0.999, 1e-8, step=step, stochastic=noisy, seed=22, stream=stream_ptr())
        torch.cuda.synchronize()
        m, ms, v, vs = state
        state = oracle.adamw_moments_fp32(host(param.g), m, ms, v, vs, 0.9, 0.999, 1.0, oracle.adamw_noise(22, step, 0, n) if noisy else None)
        for name, got, want in zip(("m", "m_scale", "v", "v_scale"), (param.m, param.ms.t, param.v, param.vs.t), state):
            assert np.array_equal(host(got), want), (step, name, int((host(got) != want).sum()))
    for b in param.guards:
        b.check()
