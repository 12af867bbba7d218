"""The limits and choices that include/ozimmu_lm.h states in numbers (host, no GPU)."""
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2409_13313_amd", "libozimmu.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libozimmu.so not built (run __graft_entry__.build())")
AT, DIM, BF16, TILE = 4096, -2, 1, 1


@pytest.fixture(scope="module")
def lib():
    pytest.importorskip("torch")
    from paper_2409_13313_amd import lm
    return lm._lib


@pytest.mark.parametrize("n,p", [(4096, 4096), (512, 1024), (4096, 1000), (2048, 300), (64, 4097), (8192, 32768), (1, 1)])
def test_weights_are_read_back_from_one_number_of_rows_on(lib, n, p):
    text = re.sub(r"\s*\n \* ", " ", open(os.path.join(ROOT, "include", "ozimmu_lm.h")).read())
    rows, power = map(int, re.search(r"takes the first up to (\d+) rows, or up to m p = 2\^(\d+) where that is more", text).groups())
    last = max(rows, 2 ** power // p)
    for m in [*range(1, 4500), last - 1, last, last + 1, 2 * last]:
        if m < 2 ** 22 - 255:
            assert (lib.ozimmu_lm_linear_choose(m, n, p) == TILE) == (m > last), m


def test_sizes_of_a_loss(lib):
    def loss(m, n, p=100):
        return lib.ozimmu_lm_cross_entropy(BF16, m, n, p, AT, n, AT, n, AT, 1, -100, AT, AT, None, 0, None)
    limit = 2 ** 31 - 2 ** 20
    for m, n in ((2 ** 22 - 256, 256), (2 ** 22 - 256, 257), (8191 * 256, 1024), (8188 * 256, 1024), (2048, 2 ** 20 - 512), (2047, 2 ** 20), (2049, 2 ** 20)):
        fits = -(-m // 256) * 256 * (-(-n // 256) * 256) < limit
        assert (loss(m, n) == DIM) == (not fits), (m, n)             # (one that fits is refused for want of a workspace)
        assert (lib.ozimmu_lm_cross_entropy_workspace_bytes(m, n, 100) > 0) == fits
        assert (lib.ozimmu_lm_cross_entropy_backward_workspace_bytes(m, n, 100) > 0) == fits
    assert loss(4, 0) == DIM and loss(4, 8, 0) == DIM
