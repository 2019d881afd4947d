"""How the matrix products are cut (hg_dense_plan.hpp), evaluated on the CPU: which sizes of the GPU tests get
which tiles, grids that the device takes for every size that the calls take, workspaces for the parts."""
import os
import shutil
import subprocess

import pytest

import paper_2112_15345_amd as hg
from paper_2112_15345_amd import dense

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")
LARGE, MEDIUM, SMALL, TALL = range(4)
F32, F16, BF16, E4M3 = 1, 2, 3, 4
MOST = (1 << 31) - 1

PROGRAM = r"""
#include <cstdio>
#include "hg_dense_plan.hpp"
using namespace hg;
int main() {
  long long rows, cols, depth; int dtype, both, direct;
  while (std::scanf("%lld %lld %lld %d %d %d", &rows, &cols, &depth, &dtype, &both, &direct) == 6) {
    const int64_t slab = slab_of(dtype);
    int n = 0;
    for (int64_t left = rows; left > 0 && ++n < 1000;) {
      const Plan p = plan_of(left, cols, depth, slab, both, direct);
      const int64_t threads = p.cut == Cut::kLarge || p.cut == Cut::kTall ? 512 : 256;
      std::printf("%d,%lld,%lld,%lld,%lld,%lld ", int(p.cut), (long long)p.rows,
                  (long long)(ceil_div(p.rows, p.tile_i) * ceil_div<int64_t>(cols, p.tile_j)),
                  (long long)threads, (long long)p.splits, (long long)p.per_split);
      if (p.rows <= 0) return 1;
      left -= p.rows;
    }
    std::printf("| %lld %d\n", (long long)parts_bytes(rows, cols, depth, slab, both),
                int(is_few(rows, cols)));
  }
}
"""


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    """plans([(rows, cols, depth, dtype, both, direct)]) -> [(launches, bytes of parts, few rows)], a
    launch (cut, rows, tiles, threads, splits, per_split)."""
    where = tmp_path_factory.mktemp("plans")
    src, exe = str(where / "plans.cpp"), str(where / "plans")
    with open(src, "w") as f:
        f.write(PROGRAM)
    res = subprocess.run(["g++", "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__=1", "-I",
                          os.path.join(ROOT, "include"), "-I",
                          os.path.join(ROOT, "paper_2112_15345_amd", "csrc"), "-isystem",
                          "/opt/rocm/include", src, "-o", exe], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr

    def run(sizes):
        text = "\n".join(" ".join(str(int(x)) for x in s) for s in sizes)
        out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout
        got = []
        for line in out.splitlines():
            launches, rest = line.split("|")
            got.append(([tuple(int(x) for x in t.split(",")) for t in launches.split()],
                        *(int(x) for x in rest.split())))
        assert len(got) == len(sizes)
        return got

    return run


def cuts(plan):
    return [launch[0] for launch in plan[0]]


def test_tiles_that_the_gpu_tests_name(plans):
    """The sizes of test_gpu_dense_tiles.py and test_gpu_dense_float32.py reach what they are there for."""
    for dt in (BF16, E4M3):
        for m, k, n in [(8201, 512, 4104), (8193, 520, 4112)]:
            (p,) = plans([(m, n, k, dt, 0, 1)])
            assert cuts(p) == [LARGE], (m, k, n)
        for m, k, n in [(8201, 1032, 8200), (12_001, 1160, 2816)]:
            (p,) = plans([(m, n, k, dt, 0, 1)])
            assert cuts(p)[0] == LARGE and len(cuts(p)) > 1, (m, k, n)
    for m, k, n in [(8201, 1032, 8200), (12_001, 1160, 2816)]:
        (p,) = plans([(m, n, k, F32, 0, 1)])
        assert cuts(p)[0] == MEDIUM
    assert len(plans([(12_001, 2816, 1160, F32, 0, 1)])[0][0]) > 1
    # backward: dx (m x k over n), dw (n x k over m)
    for m, k, n in [(8201, 4104, 520), (8201, 4104, 1032), (8193, 8200, 1040)]:
        dx, dw = plans([(m, k, n, BF16, 0, 1), (n, k, m, BF16, 1, 1)])
        assert cuts(dx)[0] == LARGE and (len(cuts(dx)) > 1) == (n >= 1024)
    assert cuts(plans([(1040, 8200, 8193, BF16, 1, 1)])[0])[0] == TALL
    # float32 on 128 x 128 tiles, which multiply by pieces
    for rows, cols, depth, both in [(2100, 1032, 72, 0), (2100, 1100, 1032, 0), (1032, 1100, 2100, 1),
                                    (20_000, 520, 8, 0), (2100, 1100, 8, 1)]:
        assert cuts(plans([(rows, cols, depth, F32, both, 1)])[0]) == [MEDIUM], (rows, cols, depth)
    # (those that are not: their values end in the 32-bit instructions)
    assert cuts(plans([(300, 136, 72, F32, 0, 1)])[0]) == [SMALL]


WILD = [1, 2, 33, 129, 1000, 70_001, (1 << 22) + 1, (1 << 27) + 5, 1 << 28, (1 << 28) + 1, (1 << 30) + 3,
        MOST - 128, MOST]


def test_grids_of_every_size(plans):
    """Every launch's grid has fewer than 2^32 threads (columns past 2^28 are taken in halves), its
    parts cover the depth, and the rows end.  Sizes are any that one array of 288 GB could have."""
    sizes = [(r, c, d, dt, both, direct) for r in WILD for c in WILD for d in (0, 1, 40, 5000, 1 << 20, MOST)
             for dt in (F32, BF16) for both in (0, 1) for direct in (0, 1)
             if c <= 1 << 28 and r * c <= 1 << 37]
    for size, (launches, parts, _) in zip(sizes, plans(sizes)):
        rows, cols, depth = size[:3]
        assert sum(launch[1] for launch in launches) == rows
        for cut, n, tiles, threads, splits, per_split in launches:
            assert 0 < tiles * threads < 1 << 32, (size, launches)
            assert 1 <= splits <= 65535 and splits * per_split >= depth
            if splits > 1:
                assert parts >= splits * n * cols * 4 and (splits - 1) * per_split < depth


def test_wide_products_have_no_parts(plans):
    """Products whose columns are taken in halves are never cut along the depth, before or after."""
    for cols in ((1 << 28) + 1, (1 << 30) + 3, MOST):
        for rows in (1, 40, 300):
            for both in (0, 1):
                (whole,) = plans([(rows, 1 << 28, MOST, BF16, both, 1)])
                assert all(launch[4] == 1 for launch in whole[0])
                half = cols // 2 // 256 * 256
                while half > 1 << 28:
                    half = half // 2 // 256 * 256
                for c in (half, 1 << 27):
                    (p,) = plans([(rows, c, MOST, BF16, both, 1)])
                    assert all(launch[4] == 1 for launch in p[0])


def test_workspaces_of_the_largest_sizes():
    """Broadcast rows may make the sizes' product pass 2^63: the bytes do not wrap around."""
    lib = hg.load_library()
    for m, k, n in ((MOST, 1, MOST), (MOST, MOST, 1), (1, MOST, MOST), (MOST, MOST, MOST)):
        for dt in (F32, BF16):
            for act in (0, 2):
                need = lib.hg_linear_grad_workspace(m, k, n, dt, act)
                assert need >= (m * n * 2 if act else 0) or need == (1 << 63) - 1
            assert lib.hg_linear_workspace(m, k, n, dt) >= 0
    # and a call that claims less is refused
    p = 0x1000
    a = dense.LinearGradArgs(m=MOST, k=1, n=MOST, dtype=F32, dw_dtype=F32, act=1, dy=p, dy_stride=0, pre=p,
                             pre_stride=0, x=p, x_stride=0, w=p, w_stride=0, dx=p, dx_stride=1, dw=p,
                             dw_stride=1, workspace=p, workspace_bytes=1 << 62)
    import ctypes
    assert lib.hg_linear_grad(ctypes.byref(a), None) == hg.HG_EINVAL
