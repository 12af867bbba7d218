"""The look that the build takes at the assembly of the tile kernels of microscaled 4-bit products (paper_2409_13313_amd/codegen.py): a mistake put
into one, or a build without one, is found (CPU only: hipcc cross-compiles)."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2409_13313_amd import build, codegen

pytestmark = pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc")


@pytest.fixture(scope="module")
def assembly(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("mx") / "gemm.s")
    pr = subprocess.run(["hipcc", *build.FLAGS, "--cuda-device-only", "-S", os.path.join(build.CSRC, "ozimmu_mx_gemm.hip"), "-o", out],
                        stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert pr.returncode == 0, pr.stdout[-3000:]
    return open(out).read()


def test_every_instance_is_looked_at(assembly):
    assert codegen.check_mx(assembly) == {"k_mx_tile": 3, "k_mx_half": 3}
    assert all(src in build.SOURCES for src in build.LOOKED_AT)


def at(lines, pattern, number=0):
    return [i for i, line in enumerate(lines) if re.search(pattern, line)][number]


def before_copy(lines):
    """a copy of the loop, and the scalar register that holds its size"""
    i = at(lines, codegen.MX_MFMA, 10)
    i = next(j for j in range(i, len(lines)) if re.search(r"buffer_load_dwordx4 .* lds", lines[j]))
    lo = int(re.search(r"s\[(\d+):", lines[i]).group(1))
    return next(j for j in range(i, 0, -1) if "#ASMSTART" in lines[j]), lo + 2


def plant_size(lines):
    i, reg = before_copy(lines)
    lines.insert(i, f"\tv_readfirstlane_b32 s{reg}, v0")


MISTAKES = {
    "a vector instruction writes the size of a copy right before it": plant_size,
    "spills": lambda lines: lines.insert(at(lines, codegen.MX_MFMA, 5), "\tscratch_store_dword off, v0, off"),
    "a wait of the compiler's in the loop": lambda lines: lines.insert(at(lines, codegen.MX_MFMA, 5), "\ts_waitcnt vmcnt(0)"),
    "another user of M0": lambda lines: lines.insert(at(lines, codegen.MX_MFMA, 5), "\ts_mov_b32 m0, s0"),
    "no wait states behind the products": lambda lines: lines.__setitem__(slice(0, len(lines)), [x.replace("s_nop 15", "s_nop 0") for x in lines]),
    "no barrier": lambda lines: lines.pop(at(lines, "s_barrier", 1)),
    "a sum moves": lambda lines: lines.insert(at(lines, codegen.MX_MFMA, 5), "\tv_accvgpr_write_b32 a3, v0"),
    "sums not in place": lambda lines: lines.__setitem__(at(lines, codegen.MX_MFMA, 3), re.sub(r"a\[\d+:\d+\]", "a[252:255]", lines[at(lines, codegen.MX_MFMA, 3)], count=1)),
    "no wait state behind a store": lambda lines: lines.pop(at(lines, "s_nop 1$", 3)),
}


@pytest.mark.parametrize("kernel", ["k_mx_tileILi1E", "k_mx_halfILi0E"])
@pytest.mark.parametrize("mistake", list(MISTAKES))
def test_a_mistake_is_found(assembly, kernel, mistake):
    m = re.search(r"^_ZN12_GLOBAL__N_1\d+" + kernel + r"\w+:.*?^\.Lfunc_end", assembly, re.S | re.M)
    lines = m.group(0).split("\n")
    MISTAKES[mistake](lines)
    with pytest.raises(codegen.Wrong):
        codegen.check_mx(assembly[:m.start()] + "\n".join(lines) + assembly[m.end():])


def test_a_build_without_one_is_found(assembly):
    with pytest.raises(codegen.Wrong):
        codegen.check_mx(assembly.replace("k_mx_halfILi2E", "k_mx_hallILi2E"))
