"""Which tiles products take, on the CPU: the planner compiled alone.  The sizes that the GPU tests run reach every tile that there is a kernel for, so
that a change of the planner's costs cannot leave one without a test."""
import os
import shutil
import subprocess

import pytest

import paper_2602_16249_amd as aff
from product_sizes import SIZES

MAIN = """
#include "linear_plan.h"
#include <cstdio>
using namespace affmae;
static int line(long long at) { return at % 16 == 0 ? 16 : at % 4 == 0 ? 4 : 2; }
int main() {
  int el, rows, cin, cout, made, off;
  while (scanf("%d %d %d %d %d %d", &el, &rows, &cin, &cout, &made, &off) == 6) {
    const auto of = [&](bool copied, int C) { return copied ? 16 : line((long long)C * el | off * el); };
    const Copies c = copies(rows, cin, cout, made, true, true, el);
    const int fwd = of(false, cin), dx = std::min(of(c.dz, cout), of(c.weight, cin)), dw = std::min(of(c.dz, cout), of(c.x, cin));
    const Plan f = plan_product(rows, cout, cin, el, fwd, true), x = plan_product(rows, cin, cout, el, dx, false), w = plan_product(cout, cin, rows, el, dw, false);
    printf("%d %d 1 %d %d %d %d %d %d\\n", fwd, f.shape, dx, x.shape, x.splits, dw, w.shape, w.splits);
  }
}
"""
TILES = ("64x64", "128x64", "128x128", "128x192", "16x16")
# type, bytes that a lane brings at a time -> tiles of a gradient; the forward has 16 x 16 too where it brings 16
KERNELS = {("bf16", 16): 4, ("bf16", 4): 3, ("bf16", 2): 3, ("f32", 16): 2, ("f32", 4): 2}


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    """f(sizes) -> per size {"fwd" | "dx" | "dweight": (bytes a lane, tile, workgroups that share k)}"""
    if shutil.which("g++") is None:
        pytest.skip("needs a host compiler")
    at = tmp_path_factory.mktemp("plan")
    (at / "main.cpp").write_text(MAIN)
    csrc = os.path.join(os.path.dirname(aff.__file__), "csrc")
    subprocess.run(["g++", "-O1", "-std=c++17", "-I", csrc, str(at / "main.cpp"), "-o", str(at / "plan")], check=True)

    def run(sizes):
        text = "\n".join(f"{4 if t == 'f32' else 2} {rows} {cin} {cout} {int(made)} {off}" for t, rows, cin, cout, made, off in sizes)
        lines = subprocess.run([str(at / "plan")], input=text, capture_output=True, text=True, check=True).stdout.split("\n")[:len(sizes)]
        out = []
        for line in lines:
            v = [int(x) for x in line.split()]
            out.append({k: (v[3 * i], TILES[v[3 * i + 1]], v[3 * i + 2]) for i, k in enumerate(("fwd", "dx", "dweight"))})
        return out

    return run


def test_the_sizes_take_every_tile(plan):
    taken = set()
    for size, got in zip(SIZES, plan(SIZES)):
        taken |= {(k, size[0], w, tile) for k, (w, tile, _) in got.items()}
    every = {(k, t, w, TILES[i]) for (t, w), n in KERNELS.items() for i in range(n) for k in ("fwd", "dx", "dweight")}
    every |= {("fwd", t, 16, "16x16") for t in ("bf16", "f32")}
    assert not every - taken, sorted(every - taken)
    assert not taken - every, sorted(taken - every)


def test_gradients_share_k_within_what_there_is(plan):
    """Slices for every workgroup that shares a tile's k, and none shared in the forward."""
    sizes = [(t, rows, cin, cout, made, off) for t in ("bf16", "f32") for rows in (1, 63, 64, 65, 130, 5000, 131072, 1 << 29) for cin, cout in ((1, 1), (3, 64), (64, 3), (40, 63))
             for made in (False, True) for off in (0, 1)]
    for size, got in zip(sizes, plan(sizes)):
        deep = 32 if size[0] == "f32" else 64
        assert got["fwd"][2] == 1
        for k, depth in (("dx", size[3]), ("dweight", size[1])):
            slices = -(-depth // deep)
            splits = got[k][2]
            assert 1 <= splits <= max(1, slices // 2)
            each = -(-slices // splits)
            assert (splits - 1) * each < slices, size  # (the last one has some too)
