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


@pytest.mark.parametrize("m,n,p", [(1, 4096, 32768), (1, 4096, 131072), (18, 253, 81303), (64, 8192, 131072), (300, 4096, 131072), (2048, 4096, 131072), (1, 2 ** 20, 1000)])
def test_the_gradients_copy_of_w(lm, m, n, p):
    """Slopes of at most 128 MB and W laid out, at most 256 MB of it; beside them X twice and the sums of the states' gradient, no more than 256 rows of it for each
    split (of which there are 256 at the most)."""
    need = lm.cross_entropy_workspace_bytes(m, n, p, backward=True)
    padded, width = -(-m // 256) * 256, -(-n // 256) * 256
    states = (256 if m < 256 else 8) * padded * width * 4
    assert need <= 128 * MB + max(256 * MB, 256 * width * 2) + 2 * m * width * 2 + min(states, 96 * MB if n < 2 ** 20 else states) + 64 * padded + SMALL


def test_many_tokens(lm):
    """From 262144 tokens on slopes are of 256 words at a time, whatever they take: 512 bytes a token."""
    for m in (262144, 1000000, 2 ** 22 - 256):
        need = lm.cross_entropy_workspace_bytes(m, 8, 10000, backward=True)
        assert need <= m * 512 + m * 256 * 4 + 3 * m * 128 + 64 * m + MB
