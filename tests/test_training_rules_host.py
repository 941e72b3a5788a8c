"""CPU-side tests of the rules by which the operators of a training step deal their work and default their arguments."""
import os
import shutil
import subprocess

import pytest

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
