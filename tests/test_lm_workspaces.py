"""What the loss and its gradient ask for as a workspace, against what they hold in it (host, no GPU): bytes of each piece as the calls use them."""
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2409_13313_amd", "libozimmu.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libozimmu.so not built (run __graft_entry__.build())")
MB = 2 ** 20
SMALL = 64 * 1024   # a few vectors of some tokens, rounded up


@pytest.fixture(scope="module")
def lm():
    pytest.importorskip("torch")
    from paper_2409_13313_amd import lm
    return lm


# tokens, elements, words, tokens a workgroup: two numbers for 16 words and each token of whole workgroups
@pytest.mark.parametrize("m,n,p,rows", [(1, 64, 2 ** 22 - 256, 16), (1, 4096, 131072, 16), (16, 64, 32768, 16)])
def test_parts_of_few_tokens(lm, m, n, p, rows):
    assert lm.cross_entropy_workspace_bytes(m, n, p) <= rows * p // 16 * 8 + SMALL


@pytest.mark.parametrize("m", [1, 16, 64, 300, 1000, 3000])
@pytest.mark.parametrize("n", [8, 64, 200])
@pytest.mark.parametrize("p", [1000, 131072, 2 ** 21 + 5, 2 ** 22 - 256])
def test_parts_are_no_more_than_they_are_said_to_be(lm, m, n, p):
    """256 MB, and W laid out, another 256 MB, and X."""
    need = lm.cross_entropy_workspace_bytes(m, n, p)
    x = -(-m // 256) * 256 * 256 * 2
    assert need <= 256 * MB + min(256 * MB, (p + 256) * 256 * 2) + x + 8 * m + SMALL
