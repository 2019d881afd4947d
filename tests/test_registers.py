"""The kernels of the built library keep what they hold in registers: spilled sums in a product's loop
give right results and take twice the time.  Read from the library's own metadata (no GPU needed)."""
import os
import re
import subprocess

import pytest

import paper_2112_15345_amd as hg

TOOLS = "/opt/rocm/llvm/bin"
OBJCOPY, BUNDLER, READELF = (os.path.join(TOOLS, t) for t in ("llvm-objcopy", "clang-offload-bundler",
                                                              "llvm-readelf"))
pytestmark = pytest.mark.skipif(
    not all(os.path.exists(p) for p in (OBJCOPY, BUNDLER, READELF, hg.LIB_PATH)),
    reason="no library, or none of the tools that read it")


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """Name -> (scratch bytes of a thread, spilled vector registers)."""
    where = tmp_path_factory.mktemp("code")
    fat, part, elf = (str(where / f) for f in ("fat", "part", "elf"))
    subprocess.run([OBJCOPY, "--dump-section", ".hip_fatbin=" + fat, hg.LIB_PATH, os.devnull],
                   check=True)
    with open(fat, "rb") as f:
        data = f.read()
    at = [m.start() for m in re.finditer(b"__CLANG_OFFLOAD_BUNDLE__", data)] + [len(data)]
    found = {}
    for first, last in zip(at, at[1:]):
        with open(part, "wb") as f:
            f.write(data[first:last])
        subprocess.run([BUNDLER, "--unbundle", "--type=o", "--input=" + part, "--output=" + elf,
                        "--targets=hipv4-amdgcn-amd-amdhsa--gfx950"], check=True)
        notes = subprocess.run([READELF, "--notes", elf], check=True, capture_output=True,
                               text=True).stdout
        for k in notes.split("\n  - .")[1:]:
            name, *figures = (re.search(p + r":\s+(\S+)", k) for p in
                              (r"\.name", "private_segment_fixed_size", "vgpr_spill_count"))
            if name and all(figures):
                found[name[1]] = tuple(int(f[1]) for f in figures)
    return found


def test_nothing_is_spilled(kernels):
    assert sum("k_product_direct" in n for n in kernels) >= 20
    # (the step of the distillation holds the longest rows that fit, and puts 3 to 7 registers away)
    spilled = {n: f for n, f in kernels.items() if any(f) and "k_distill_step" not in n}
    assert not spilled
