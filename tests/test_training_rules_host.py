"""CPU-side tests of the rules by which the operators of a training step deal their work, default their arguments and round with noise."""
import os
import shutil
import subprocess

import numpy as np
import pytest

import oracle

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2511_21089_b200", "csrc")

# Evaluated by the compiler, which takes no access outside of a table: each (first, last, step) is a range of row lengths.
SHAPES = """
#include <initializer_list>

#include "norm_shapes.h"
using namespace mlpmoe;
constexpr bool holds(int64_t first, int64_t last, int64_t step) {
  for (int64_t d = first; d <= last; d += step) {
    const int s = shape_of(d);
    if (s < 0 || s > kLastShape) return false;
    if (d <= kOnePassD && kShapes[s].threads * 8 < d) return false;              // a thread for every column
    if (s > 0 && kShapes[s - 1].threads * 8 >= d) return false;                  // and no smaller shape has them
    for (int64_t n : {int64_t{0}, int64_t{1}, int64_t{63}, int64_t{64}, int64_t{149}, int64_t{592}, int64_t{16384}, int64_t{2147483647}}) {
      const int64_t blocks = blocks_of(n, d);
      if (blocks < 0 || blocks > n || (n > 0 && blocks == 0)) return false;
      if (d > kOnePassD && blocks != (n < kSplitRows ? n : kSplitRows)) return false;
      if (d <= kOnePassD && blocks > int64_t{kSms} * kShapes[s].ctas) return false;
    }
  }
  return true;
}
static_assert(holds(%d, %d, %d), "a row length without a shape, or blocks without rows");
int main() { return 0; }
"""


@pytest.mark.parametrize("first,last,step", [(1, 2100, 1), (2101, 8192, 7), (8185, 8192, 1), (8193, 8400, 1), (8193, 32768, 61), (32760, 32768, 1)])
def test_norm_gradient_shapes_of_every_row_length(tmp_path, first, last, step):
    compiler = shutil.which("g++") or shutil.which("c++")
    assert compiler, "the extension is built with a C++ compiler"
    source = tmp_path / "shapes.cpp"
    source.write_text(SHAPES % (first, last, step))
    r = subprocess.run([compiler, "-std=c++17", "-fconstexpr-ops-limit=1000000000", "-fconstexpr-loop-limit=1000000", "-fsyntax-only", "-I", CSRC, str(source)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]


def test_a_norm_and_its_gradient_have_the_same_default_eps(lib, monkeypatch):
    seen = {}

    def taken(name, at):
        def call(*args):
            seen[name] = args[at]
            return lib.MLPMOE_OK
        monkeypatch.setattr(lib.lib, name, call)
    for name in ("mlpmoe_add_rmsnorm", "mlpmoe_add_layernorm"):
        taken(name, -2)                                  # eps, stream
    taken("mlpmoe_norm_backward", -4)                    # eps, workspace, its bytes, stream
    for norm, forward, name in ((lib.MLPMOE_RMSNORM, lib.mlpmoe_add_rmsnorm, "mlpmoe_add_rmsnorm"),
                                (lib.MLPMOE_LAYERNORM, lib.mlpmoe_add_layernorm, "mlpmoe_add_layernorm")):
        forward(0x10000, None, 0x20000, 0x30000, 4, 64)
        lib.mlpmoe_norm_backward(norm, 0x20000, 0x40000, 0x50000, 4, 64)
        assert seen["mlpmoe_norm_backward"] == seen[name]
        lib.mlpmoe_norm_backward(norm, 0x20000, 0x40000, 0x50000, 4, 64, eps=0.25)
        assert seen["mlpmoe_norm_backward"] == 0.25


# ----------------------------------------------------------------------------- params in bf16, rounded with noise

def test_bf16_rounding_pins():
    """The added bits are the low half of mix32(noise ^ 0x9E3779B1), and what is left below bf16 is cut off."""
    for noise in (0, 1, 0x12345678, 0xFFFFFFFF):
        low = oracle.mix32(noise ^ 0x9E3779B1) & 0xFFFF
        for sign in (0, 0x80000000):
            for cut, up in ((0, 0), (65535 - low, 0), (65536 - low, 1 if low else None), (65535, 1 if low else 0)):
                if up is None:
                    continue
                bits = np.array([sign | 0x3F800000 + cut], np.uint32)
                want = np.array([sign | 0x3F800000 + 0x10000 * up], np.uint32).view(np.float32)[0]
                assert oracle.bf16_up_or_down(bits.view(np.float32).astype(np.float64), [noise])[0] == want, (noise, sign, cut)


@pytest.mark.parametrize("p", [1.0, 1.0 + 2.0 ** -9, -1.003, 0.0199, 3e-5, -127.6])
def test_bf16_rounding_has_the_right_mean(p):
    noise = oracle.adamw_noise(5, 1, 0, 100000)
    got = oracle.bf16_up_or_down(np.full(100000, p), noise)
    p = float(np.float32(p))
    step = 2.0 ** (np.floor(np.log2(abs(p))) - 7)
    assert set(np.unique(np.abs(got))) <= {np.floor(abs(p) / step) * step, (np.floor(abs(p) / step) + 1) * step}
    # a coin of deviation step / 2 at most, 100000 times
    assert abs(got.mean() - p) <= 5 * step / 2 / np.sqrt(100000)


def test_other_roundings_to_bf16_are_told_apart():
    """Truncation, away from zero, to nearest, and other words of the noise give another neighbour for a fifth of the elements or more."""
    rng = np.random.default_rng(6)
    p, noise = (rng.normal(size=20000) * 0.02).astype(np.float32), oracle.adamw_noise(6, 2, 1, 20000)
    want = oracle.bf16_up_or_down(p, noise)
    bits = p.view(np.uint32).astype(np.uint64)

    def plus(extra):
        return ((bits + np.asarray(extra, np.uint64)) & np.uint64(0xFFFF0000)).astype(np.uint32).view(np.float32)
    mixed = np.array([oracle.mix32(int(h) ^ 0x9E3779B1) for h in noise], np.uint64)
    others = {"truncated": plus(0), "away": plus(0xFFFF), "nearest": plus(0x7FFF), "unmixed": plus(noise & np.uint64(0xFFFF)),
              "high half": plus(mixed >> np.uint64(16))}
    for name, other in others.items():
        # two independent coins of the same odds differ for 2 q (1 - q), a third on average; nearest and a coin for a quarter
        assert np.mean(other != want) > 0.2, name
    assert abs(np.mean((np.abs(want) - np.abs(p)) / 2.0 ** (np.floor(np.log2(np.abs(p))) - 7))) < 5 * 0.5 / np.sqrt(20000)
    assert np.mean((np.abs(others["truncated"]) - np.abs(p)) / 2.0 ** (np.floor(np.log2(np.abs(p))) - 7)) < -0.4


# ----------------------------------------------------------------------------- the sorted order of many tokens

@pytest.mark.parametrize("n,B,slots,align", [(1, 1, 1, 1), (70, 9, 2, 4), (200, 256, 300, 16), (333, 3, 1, 128)])
def test_sorted_order_a_branch_at_a_time(n, B, slots, align):
    rng = np.random.default_rng([n, B])
    select = (rng.uniform(size=(n, B)) < 0.4).astype(np.uint8) * rng.integers(1, 256, (n, B)).astype(np.uint8)
    want, got = oracle.sort_tokens(select, slots, align), oracle.sort_tokens_of_many(select, slots, align)
    assert all(np.array_equal(want[name], got[name]) for name in want)


def test_sort_workspace_serves_smaller_batches_past_the_largest_tiles(lib):
    """Batches on both sides of the size from which tiles no longer grow and more of them are made."""
    for B, most in ((3, 32), (64, 32), (128, 32), (129, 25), (200, 18), (256, 16)):
        at = 592 * most * 32
        sizes = [lib.mlpmoe_sort_workspace(n, B) for n in list(range(at - 64 * 31, at + 64 * 31, 31)) + [2 * at, 5 * at]]
        assert sizes == sorted(sizes)
        B32 = -(-B // 32) * 32
        for n, size in ((at, sizes[64]), (2 * at, sizes[-2])):
            groups = -(-n // 32)
            assert size >= groups * B32 * 4 + (-(-groups // most) + 1) * B32 * 4      # the bits, and the tiles' counts with their totals


# ----------------------------------------------------------------------------- the list of an optimizer step

def test_a_list_of_tensors_takes_addresses_and_new_gradients(lib):
    import gc
    import weakref

    import torch
    p, g, m, v = (torch.zeros(8) for _ in range(4))
    tensors = lib.mlpmoe_adamw_tensors([dict(n=8, param=p, grad=g.data_ptr(), m=m, v=v)])
    gone, address = weakref.ref(g), g.data_ptr()
    assert tensors[0].grad == address and tensors[0].param == p.data_ptr()
    del g
    gc.collect()
    assert gone() is None                                  # an address keeps no tensor
    kept = weakref.ref(m)
    del m
    gc.collect()
    assert kept() is not None                              # a tensor is kept
    new = torch.zeros(8)
    tensors[0].grad = new.data_ptr()
    assert tensors[0].grad == new.data_ptr() and tensors[0].m == kept().data_ptr() and tensors[0].n == 8


# ----------------------------------------------------------------------------- 8-bit moments bit by bit

@pytest.mark.parametrize("noisy", [False, True])
def test_moments_bit_by_bit_are_those_of_the_definition(noisy):
    """The fp32 arithmetic against 64 bits: scales within its roundings, codes the same but next to a border."""
    rng = np.random.default_rng(17)
    n = 128 * 150 + 37
    (m, ms), (v, vs) = oracle.adamw_blocks(rng.normal(size=n) * 3e-4, False), oracle.adamw_blocks(np.abs(rng.normal(size=n)) * 1e-3, True)
    ms, vs = ms.astype(np.float32), vs.astype(np.float32)
    g = (rng.normal(size=n) * 1e-3).astype(np.float32)
    noise = oracle.adamw_noise(3, 5, 0, n) if noisy else None
    cm, sm, cv, sv = oracle.adamw_moments_fp32(g, m, ms, v, vs, 0.9, 0.999, 0.37, noise)
    _, m1, v1 = oracle.adamw(0.0, g.astype(np.float64), m * np.repeat(ms, 128)[:n].astype(np.float64),
                             (v * np.repeat(vs, 128)[:n].astype(np.float64)) ** 2, 1e-3, 0.9, 0.999, 1e-8, 0.0, 5, float(np.float32(0.37)))
    u = 2.0 ** -24
    for x, root, codes, scales in ((m1, False, cm, sm), (np.sqrt(v1), True, cv, sv)):
        want, want_scale = oracle.adamw_blocks(x, root, noise)
        # constants, products and the sum 5 u of the terms (a sum of two that cancel: the block's largest does not), root and product 2 u each
        assert np.all(np.abs(scales - want_scale) <= 12 * u * want_scale)
        assert np.mean(codes != want) <= 2e-3
        assert np.all(np.abs(codes - want) <= 2.0 ** -3 * np.maximum(np.abs(want), 2.0 ** -6))
