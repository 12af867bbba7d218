"""Matrices whose last element lies further from the first than any address can: refused before a launch (host, no GPU).  The least of them are
looked at; the largest that are allowed are larger than any memory."""
import os

import pytest

torch = pytest.importorskip("torch")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2409_13313_amd", "libozimmu.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libozimmu.so not built (run __graft_entry__.build())")

DIM = -2
AT = 4096            # an address that is never looked at
F32, BF16 = 0, 1
MOST_ROWS, MOST_INNER, MOST_LD = 2 ** 22 - 256, 2 ** 29, 2 ** 40 - 1


@pytest.fixture(scope="module")
def lib():
    from paper_2409_13313_amd import mx
    return mx._lib


@pytest.mark.parametrize("kind", [F32, BF16])
def test_rows_times_leading_dimension(lib, kind):
    """rows x leading dimension stays below 2^60 elements, so that every offset in bytes fits 64 bits."""
    # by columns alone: as many rows as an inner dimension has positions
    for rows, ld in ((MOST_INNER, MOST_LD), (MOST_INNER, 2 ** 31), (2 ** 21, 2 ** 39), (MOST_ROWS, 2 ** 39)):
        assert rows * ld >= 2 ** 60
        assert lib.ozimmu_mx_quantize(kind, rows, 4, AT, ld, None, AT, None) == DIM
    rows, ld = MOST_ROWS, MOST_LD
    assert lib.ozimmu_mx_quantize(kind, rows, 4, AT, ld, AT, None, None) == DIM
    assert lib.ozimmu_mx_dequantize(kind, rows, 4, AT, AT, ld, None) == DIM
    assert lib.ozimmu_mx_gemm(rows, 4, 4, 1.0, AT, AT, 0.0, kind, AT, ld, None) == DIM
    room = lib.ozimmu_mx_workspace_bytes(rows, 4, 4)
    for ldx, ldd in ((ld, 4), (4, ld)):
        assert lib.ozimmu_mx_linear(rows, 4, 4, 1.0, kind, AT, ldx, AT, 0.0, kind, AT, ldd, AT, room, None) == DIM
    room = lib.ozimmu_mx_backward_workspace_bytes(rows, 4, 4)
    for ldg, ldx, lddx in ((ld, 4, 4), (4, ld, 4), (4, 4, ld)):
        assert lib.ozimmu_mx_linear_backward(rows, 4, 4, 1.0, kind, AT, ldg, AT, ldx, AT, 0.0, kind, AT, lddx, 0.0, F32, AT, 4, AT, room, None) == DIM
    room = lib.ozimmu_mx_backward_workspace_bytes(4, 4, rows)
    assert lib.ozimmu_mx_linear_backward(4, 4, rows, 1.0, kind, AT, rows, AT, 4, None, 0.0, kind, None, 0, 0.0, F32, AT, ld, AT, room, None) == DIM


def test_what_has_no_rows_or_one_is_not_refused_for_its_leading_dimension(lib):
    assert lib.ozimmu_mx_quantize(F32, 0, 4, None, MOST_LD, None, None, None) == 0
    assert lib.ozimmu_mx_gemm(0, 4, 4, 1.0, None, None, 0.0, F32, None, MOST_LD, None) == 0
    # (a null pointer is found behind the sizes)
    assert lib.ozimmu_mx_quantize(F32, 1, 4, None, MOST_LD, AT, None, None) == -1
    assert lib.ozimmu_mx_quantize(F32, 2 ** 19, 4, None, MOST_LD, AT, None, None) == -1
