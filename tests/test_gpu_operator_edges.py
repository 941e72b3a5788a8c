"""GPU tests of the operators around a routed layer step where a call is allowed but unusual: long rows on small groups, values
that are not finite, sums of counts past 32 bits, calls from two host threads, weights that no token uses."""
import threading

import numpy as np
import pytest
import torch

import oracle
from tests.helpers import stream_ptr
from tests.test_gpu_operators import PATHS, TORCH, U, W4Case, dev, host, kind

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------ 4-bit layer

@pytest.mark.parametrize("group", [32, 64])
@pytest.mark.parametrize("d,d_b", [(51328, [64, 80]), (53248, [96, 48]), (65536, [64, 80]), (136, [51312, 16]), (128, [53232, 16]), (128, [65520, 16])])
def test_w4_forward_long_rows_on_small_groups(lib, d, d_b, group):
    """Rows whose digits, units and rings do not fit in shared memory together: few tokens take the tiled kernels then."""
    c = W4Case(lib, [81, d, group], d, d_b, group, True, std=0.02)
    for n, yt in ((1, "fp32"), (1, "bf16"), (5, "fp32"), (8, "bf16"), (8, "fp32"), (11, "fp32")):
        xh, x, _ = c.activations([82, n], n, "bf16")
        c.check(c.run(x, n, "bf16", yt), xh, "bf16", yt)
        sel = np.zeros((n, 2), np.uint8)
        sel[:, 0] = 1
        sel[0, 1] = 1
        c.check(c.run(x, n, "bf16", yt, select=torch.from_numpy(sel).cuda()), xh, "bf16", yt, sel)


# every path with every type of y that it takes: (d_model, branch widths, tokens, type of y)
EVERY = {"stream fp32": (520, [96, 160, 256], 5, "fp32"), "stream bf16": (520, [96, 160, 256], 7, "bf16"), "tiled fp32": (520, [96, 160, 256], 40, "fp32"),
         "tiled bf16": (520, [96, 160, 256], 40, "bf16"), "tensor": PATHS["tensor"]}


@pytest.mark.parametrize("path", list(EVERY))
@pytest.mark.parametrize("group", [32, 64, 128])
def test_w4_forward_values_that_are_not_finite(lib, path, group):
    """A NaN or an infinity in a live token's x, or an intermediate activation past fp32's range, shows in all of the token's y; the
    other tokens keep their bits."""
    d, d_b, n, yt = EVERY[path]
    c = W4Case(lib, [83, group], d, d_b, group, False, std=0.05)
    for xt, bad in (("bf16", (float("nan"), float("inf"), float("-inf"))), ("fp32", (float("nan"), float("inf"), 1e30)), ("e4m3", (float("nan"),))):
        _, x, sc = c.activations([84], n, xt)
        want = c.run(x, n, xt, yt, sc).clone()
        for k, value in enumerate(bad):
            row, wide = (0, n - 1, 2)[k], x.float().clone()
            if value == 1e30:
                wide[row] *= value                      # finite x and gates, but their product is not
            else:
                wide[row, (d - 1, 37, 0)[k]] = value
            broken = torch.empty_like(x)
            broken.copy_(wide)
            got = c.run(broken, n, xt, yt, sc)
            rest = torch.arange(n, device="cuda") != row
            assert not bool(torch.isfinite(got[row].float()).any()), (xt, value)
            assert torch.equal(got[rest], want[rest]), (xt, value)


@pytest.mark.parametrize("path", list(EVERY))
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("group,x_group", [(32, 0), (32, 64), (128, 128)])
def test_w4_forward_scales_of_x_that_are_not_finite(lib, path, value, group, x_group):
    """A scale of 8-bit activations that is NaN or infinite shows in all of the token's y, also over codes that are all 0."""
    d, d_b, n, yt = EVERY[path]
    c = W4Case(lib, [92, group], d, d_b, group, True, std=0.05)
    _, x, sc = c.activations([93], n, "e4m3", x_group)
    want = c.run(x, n, "e4m3", yt, sc, x_group).clone()
    zeros, broken = x.view(torch.uint8).clone().view(x.dtype), sc.clone()
    last = broken.shape[1] - 1
    broken[1, last], broken[n - 1, 0] = value, value
    zeros.view(torch.uint8)[n - 1, :x_group or d] = 0
    zeros.view(torch.uint8)[1, last * x_group:] = 0
    got = c.run(zeros, n, "e4m3", yt, broken, x_group)
    rest = torch.ones(n, dtype=torch.bool, device="cuda")
    rest[1] = rest[n - 1] = False
    assert not bool(torch.isfinite(got[~rest].float()).any()) and torch.equal(got[rest], want[rest])


@pytest.mark.parametrize("path", list(EVERY))
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("group", [32, 128])
def test_w4_forward_down_weights_that_a_token_does_not_use(lib, path, value, group):
    """W_down's scales of a branch are not finite: tokens without the branch are as if it were not there, tokens with it are not
    finite; and a branch with alpha = 0 stays out without a selection."""
    d, d_b, n, yt = {"stream": (200, [96, 32, 128, 256], 6, path[7:]), "tiled": (200, [96, 32, 128, 256], 40, path[6:]),
                     "tensor": (1032, [4448, 160, 4352, 128], 66, "bf16")}[path.split()[0]]
    off = oracle.branch_offsets(d_b)
    assert off[1] % 32 == 0 and off[2] % 128 == 0
    c = W4Case(lib, [85, group], d, d_b, group, True, std=0.05)
    dead = 1 if group == 32 else 3                       # one inside blocks of 128 columns that others use too; one of its own
    xh, x, _ = c.activations([86], n, "bf16")
    sel = (np.random.default_rng(87).uniform(size=(n, 4)) < 0.5).astype(np.uint8)
    sel[:, 0] |= 1                                       # every token uses the blocks around the branch
    sel[:, 2] |= 1
    none = sel.copy()
    none[:, dead] = 0
    sel[:, dead] = np.arange(n) % 2
    c.mats[2][1][off[dead] // group:off[dead + 1] // group] = value
    c.check(c.run(x, n, "bf16", yt, select=torch.from_numpy(none).cuda()), xh, "bf16", yt, none, fp16=path == "tensor")
    got = c.run(x, n, "bf16", yt, select=torch.from_numpy(sel).cuda())
    assert not bool(torch.isfinite(got[1::2].float()).any())
    r = oracle.w4_layer_forward(xh[0::2], *c.W, d_b, None, sel[0::2])
    tol = c.tolerance(r, xh[0::2], yt, "bf16" if path == "tensor" else None) + (2.0 ** -8 if yt == "bf16" else 0.0) * np.abs(r["y"])
    assert np.all(np.abs(host(got)[0::2] - r["y"]) <= tol + 1e-30)
    c.alpha = [1.0, 1.0, 0.7, 1.0]
    c.alpha[dead] = 0.0
    c.layer = lib.mlpmoe_w4_layer(d, c.I, d_b, group, *c.mats, alpha=c.alpha)
    c.check(c.run(x, n, "bf16", yt), xh, "bf16", yt, fp16=path == "tensor")


@pytest.mark.parametrize("n,yt", [(1, "bf16"), (2, "fp32"), (12, "bf16"), (12, "fp32")])
def test_w4_forward_from_two_threads(lib, n, yt):
    """Layers of two sizes that run the same kernels, called from two host threads at once, on a stream and a workspace each."""
    cases = [W4Case(lib, [88], 2048, [4096], 64, False, std=0.05), W4Case(lib, [89], 264, [64, 64], 64, False, std=0.05)]
    jobs = []
    for c in cases:
        size = lib.mlpmoe_w4_workspace(c.layer, n)
        x = c.activations([90], n, "bf16")[1].contiguous()
        y, ws = torch.empty(n, c.d, device="cuda", dtype=TORCH[yt]), torch.empty(size, device="cuda", dtype=torch.uint8)
        jobs.append((c, x, y, ws, size, torch.cuda.Stream(), c.run(x, n, "bf16", yt).clone()))
    torch.cuda.synchronize()
    failures, start = [], threading.Barrier(2)

    def work(c, x, y, ws, size, stream, want):
        try:
            start.wait()
            for _ in range(4000):
                lib.mlpmoe_w4_forward(c.layer, x, y, n, ws, size, y_dtype=kind(lib, yt), stream=stream.cuda_stream)
        except Exception as e:
            failures.append(e)
    threads = [threading.Thread(target=work, args=j) for j in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not failures
    for c, x, y, ws, size, stream, want in jobs:
        assert torch.equal(y, want)


# ------------------------------------------------------------------------------------------------ router

@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n,B", [(5, 3), (9, 32), (3, 256)])
def test_route_gradient_of_counts_past_32_bits(lib, n, B, dtype):
    """The counts of all branches may add up to more than 2^31 (2^24 tokens on 128 of 256 branches)."""
    rng = np.random.default_rng([91, B])
    logits = dev(rng.normal(size=(n, B)), dtype)
    routed = (1 << 31) - 5
    counts = np.append(rng.integers(int(0.6 * routed), routed, size=B), routed)
    assert counts[:-1].sum() > 1 << 31
    grad = torch.empty(n, B, device="cuda", dtype=TORCH[dtype])
    scale = 2.0 ** 31                                    # the gradient's 1 / T, so that bf16's smallest values play no part
    lib.mlpmoe_route_backward(logits, torch.from_numpy(counts.astype(np.int32)).cuda(), grad, n, B, grad_loss=dev([scale]), dtype=kind(lib, dtype),
                              stream=stream_ptr())
    lh = host(logits)
    want, size = oracle.route_grad(lh, counts, grad_loss=scale)
    # as check_route of the other file: x - max (span u), expf, the row's sum, a reciprocal and a product, twice; a dot product of B terms
    rel = (float(lh.max() - lh.min()) + 20) * U
    assert np.all(np.abs(host(grad) - want) <= (2 * rel + (B + 20) * U) * size + (2.0 ** -8 if dtype == "bf16" else 0.0) * np.abs(want) + 1e-38)
    assert np.abs(want).max() > 0
