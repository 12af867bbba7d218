"""The look that the build takes at the assembly of the 16-bit product tiles (paper_2409_13313_amd/codegen.py): a mistake put into one, or a build without
one, is found (CPU only: hipcc cross-compiles)."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2409_13313_amd import build, codegen

pytestmark = pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc")
MFMA = "v_mfma_f32_16x16x32_"


@pytest.fixture(scope="module")
def assembly(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("lm") / "tile.s")
    pr = subprocess.run(["hipcc", *build.FLAGS, "-DLM_TYPE=2", "--cuda-device-only", "-S", os.path.join(build.CSRC, "ozimmu_lm_tile.hip"), "-o", out],
                        stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert pr.returncode == 0, pr.stdout[-3000:]
    return open(out).read()


def test_every_instance_is_looked_at(assembly):
    assert set(codegen.check_lm(assembly, 2)) == {(k, a, b) for k in range(5) for a, b in ((8, 8), (4, 8), (4, 4))}
    assert build.LM_TYPES == (1, 2)


def at(lines, pattern, number=0):
    return [i for i, line in enumerate(lines) if re.search(pattern, line)][number]


def in_loop(lines):
    return at(lines, MFMA, -20)


def plant_size(lines):
    i = next(j for j in range(in_loop(lines), 0, -1) if re.search(r"buffer_load_dwordx4 .* lds", lines[j]))
    lo = int(re.search(r"s\[(\d+):", lines[i]).group(1))
    lines.insert(next(j for j in range(i, 0, -1) if "#ASMSTART" in lines[j]), f"\tv_readfirstlane_b32 s{lo + 2}, v0")


def drop_barrier(lines):
    begin = next(j for j in range(in_loop(lines), 0, -1) if lines[j].startswith(".LBB"))
    lines.pop(begin + at(lines[begin:], "s_barrier"))


MISTAKES = {
    "a vector instruction writes the size of a copy right before it": plant_size,
    "spills": lambda lines: lines.insert(in_loop(lines), "\tscratch_store_dword off, v0, off"),
    "a wait of the compiler's in the loop": lambda lines: lines.insert(in_loop(lines), "\ts_waitcnt vmcnt(0)"),
    "another user of M0": lambda lines: lines.insert(in_loop(lines), "\ts_mov_b32 m0, s0"),
    "no wait states behind the products": lambda lines: lines.__setitem__(slice(0, len(lines)), [x.replace("s_nop 15", "s_nop 0") for x in lines]),
    "no barrier": drop_barrier,
    "a sum moves": lambda lines: lines.insert(in_loop(lines), "\tv_accvgpr_write_b32 a3, v0"),
    "a load of the compiler's in the loop": lambda lines: lines.insert(in_loop(lines), "\tglobal_load_dword v0, v[0:1], off"),
}


@pytest.mark.parametrize("kernel", ["k_lm_tileILi2ELi1ELi8ELi8E", "k_lm_tileILi2ELi4ELi4ELi4E"])
@pytest.mark.parametrize("mistake", list(MISTAKES))
def test_a_mistake_is_found(assembly, kernel, mistake):
    m = re.search(r"^_ZN12_GLOBAL__N_1\d+" + kernel + r"\w+:.*?^\.Lfunc_end", assembly, re.S | re.M)
    lines = m.group(0).split("\n")
    MISTAKES[mistake](lines)
    with pytest.raises(codegen.Wrong):
        codegen.check_lm(assembly[:m.start()] + "\n".join(lines) + assembly[m.end():], 2)


def test_a_build_without_one_or_of_another_type_is_found(assembly):
    with pytest.raises(codegen.Wrong):
        codegen.check_lm(assembly.replace("k_lm_tileILi2ELi3ELi4ELi8E", "k_lm_tilfILi2ELi3ELi4ELi8E"), 2)
    with pytest.raises(codegen.Wrong):
        codegen.check_lm(assembly, 1)
