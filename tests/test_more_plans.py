"""How a table's gradient is cut (embed_plan in hg_dense_plan.hpp) and how integers' products are,
evaluated on the CPU: digits that cover the ids, chunks that cover the positions, arrays of the workspace
that do not overlap, grids that the device takes, integer depths that tiles take whole."""
import os
import shutil
import subprocess

import pytest

import paper_2112_15345_amd as hg

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")
MOST = (1 << 31) - 1

PROGRAM = r"""
#include <cstdio>
#include "hg_dense_plan.hpp"
using namespace hg;
int main() {
  long long n, nodes, dim;
  std::printf("%lld %lld\n", (long long)slab_of(HG_DT_I8), (long long)size_of(HG_DT_I8));
  while (std::scanf("%lld %lld %lld", &n, &nodes, &dim) == 3) {
    const EmbedPlan p = embed_plan(n, nodes, dim);
    std::printf("%d %d %d %d %lld %lld %lld %lld %lld %lld %lld %lld %lld %lld\n", p.bits, p.passes,
                p.digit, int(p.small), (long long)p.tiles, (long long)p.chunk, (long long)p.chunks,
                (long long)p.pairs, (long long)p.other, (long long)p.counts, (long long)p.totals,
                (long long)p.ends, (long long)p.parts, (long long)p.total);
  }
}
"""
SIZES = [(n, nodes, dim) for n in (1, 2, 4095, 4096, 4097, 65_537, 262_144, 262_145, 1 << 24, MOST)
         for nodes in (1, 2, 255, 256, 2047, 2048, 50_001, 1 << 22, MOST)
         for dim in (1, 16, 1024, 2048, 100_000)]


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    where = tmp_path_factory.mktemp("plans")
    src, exe = str(where / "plans.cpp"), str(where / "plans")
    with open(src, "w") as f:
        f.write(PROGRAM)
    res = subprocess.run(["g++", "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__=1", "-I",
                          os.path.join(ROOT, "include"), "-I",
                          os.path.join(ROOT, "paper_2112_15345_amd", "csrc"), "-isystem",
                          "/opt/rocm/include", src, "-o", exe], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    text = "\n".join(f"{n} {v} {d}" for n, v, d in SIZES)
    out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout
    return [[int(x) for x in line.split()] for line in out.splitlines()]


def test_embed_plans(plans):
    assert len(plans) == len(SIZES) + 1
    for (n, nodes, dim), p in zip(SIZES, plans[1:]):
        bits, passes, digit, small, tiles, chunk, chunks, pairs, other, counts, totals, ends, parts, \
            total = p
        assert nodes < 1 << bits <= 2 * nodes  # (an id that counts for nothing is `nodes`)
        assert passes * digit >= bits and digit <= (8 if small else 11)
        assert small == (n <= 4096) and (tiles - 1) * 4096 < n <= tiles * 4096
        assert 8 <= chunk <= 64 and (chunks - 1) * chunk < n <= chunks * chunk
        # pairs, the sort's other array, its counts and totals, the runs' ends, the parts
        sizes = [8 * n, 0 if small else 8 * n, 0 if small else (tiles << digit) * 4,
                 0 if small else 4 << digit, 4 * chunks, 2 * chunks * dim * 4]
        at = [pairs, other, counts, totals, ends, parts, total]
        assert at[0] == 0 and all(a % 16 == 0 for a in at[:-1])
        assert all(a + s <= b for a, s, b in zip(at, sizes, at[1:]))
        # grids of fewer than 2^32 threads, of 1024 in a block, the pieces to fill (2^21) among them
        assert (tiles + (1 << 21)) * 1024 < 1 << 32
        assert hg.load_library().hg_embed_grad_workspace(n, nodes, dim) == total


def test_integers_fill_a_slab(plans):
    """128 elements of a byte: what a tile's slab holds, so that parts begin at whole ones."""
    assert plans[0] == [128, 1]
