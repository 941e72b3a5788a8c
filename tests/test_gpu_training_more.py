"""GPU tests of the operators of a training step, beside tests/test_gpu_training.py: bf16 params rounded with noise."""
import numpy as np
import pytest
import torch

import oracle
from tests.helpers import stream_ptr
from tests.test_gpu_operators import TORCH, U, dev, host
from tests.test_gpu_training import TINY, Param

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
