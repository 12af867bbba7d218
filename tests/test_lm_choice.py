"""How the operators around the output layer are run, at sizes of which the ways are measured, and what workspace they ask for (host, no GPU)."""
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2409_13313_amd", "libozimmu.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libozimmu.so not built (run __graft_entry__.build())")

DIRECT, TILE, SHARED = 0, 1, 2


@pytest.fixture(scope="module")
def lm():
    pytest.importorskip("torch")
    from paper_2409_13313_amd import lm
    return lm


# (microseconds: straight from the codes, X in LDS, weights read back)
@pytest.mark.parametrize("m,n,p,way", [(16, 4096, 4096, DIRECT),         # 7.7  10.5
                                       (16, 8192, 16384, DIRECT),        # 18   24
                                       (128, 512, 512, DIRECT),          # 5.6  6.9
                                       (64, 4096, 4096, SHARED),         # 19   14    55
                                       (256, 1024, 16384, SHARED),       # 46   22    38
                                       (512, 4096, 4096, SHARED),        # 49   34    52
                                       (2048, 4096, 4096, TILE),         # -    90    75
                                       (4096, 4096, 16384, TILE)])       # -    630   460
def test_the_way_of_a_layer(lm, m, n, p, way):
    assert lm._lib.ozimmu_lm_linear_choose(m, n, p) == way


def test_workspaces(lm):
    assert lm.DIRECT_ROWS == 16
    for m, n, p in ((1, 1, 1), (16, 2 ** 20, 2 ** 22 - 256), (16, 4096, 4096)):
        assert lm.linear_workspace_bytes(m, n, p) == 0               # (what the binding does not ask for)
    assert lm.linear_workspace_bytes(700, 4096, 4096, "direct") == 0
    # weights read back, no more than 128 MB at a time, and X with rows of whole stages
    assert lm.linear_workspace_bytes(700, 1000, 1001, "tile") == 1024 * 1024 * 2 + 700 * 1024 * 2
    assert lm.linear_workspace_bytes(300, 4096, 131072, "tile") == 2 ** 27 + 300 * 4096 * 2
    assert lm.linear_workspace_bytes(300, 64, 10 ** 9) == 0 and lm.linear_workspace_bytes(-1, 64, 64) == 0
    # the gradient's slopes stay within 128 MB whatever the vocabulary is, the loss keeps two numbers for 64 words
    assert lm.cross_entropy_workspace_bytes(4096, 4096, 2 ** 21, backward=True) < 2 ** 29
    assert lm.cross_entropy_workspace_bytes(4096, 4096, 2 ** 21) < 2 ** 30
    for backward in (False, True):
        assert lm.cross_entropy_workspace_bytes(0, 64, 64, backward) == 0 and lm.cross_entropy_workspace_bytes(4, 64, 0, backward) == 0
        assert lm.cross_entropy_workspace_bytes(1, 1, 1, backward) > 0
