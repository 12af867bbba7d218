"""How a product of microscaled 4-bit matrices is run, at shapes of which all ways are measured (host, no GPU)."""
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2409_13313_amd", "libozimmu.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libozimmu.so not built (run __graft_entry__.build())")

DIRECT, TILE, HALF = 0, 1, 2


@pytest.fixture(scope="module")
def mx():
    pytest.importorskip("torch")
    from paper_2409_13313_amd import mx
    return mx


# (microseconds: direct, 256 x 128 tiles, 256 x 256 tiles)
@pytest.mark.parametrize("m,n,p,way", [(256, 4096, 4096, DIRECT),        # 6.8  16.8  24.9
                                       (2048, 4096, 4096, HALF),         # 32.7 21.5  27.0
                                       (4096, 4096, 4096, TILE),         # 66   39.0  36.2
                                       (1024, 8192, 8192, HALF),         # 60   35.0  44.3
                                       (2048, 8192, 8192, TILE),         # 117  68    59
                                       (512, 1024, 8192, HALF),          # 9.8  8.6   11.7
                                       (256, 1024, 8192, DIRECT),        # 5.7  8.4   11.7
                                       (2048, 1024, 8192, TILE),         # 30.9 15.4  13.9
                                       (512, 4096, 14336, HALF),         # 33.6 19.5  27.6
                                       (1024, 4096, 14336, TILE),        # 61   36.0  31.2
                                       (2048, 2051, 1283, DIRECT),       # 12.4 15.6  24.7
                                       (8192, 8192, 16384, TILE)])       # -    518   447
def test_choice(mx, m, n, p, way):
    assert mx._lib.ozimmu_mx_choose(m, n, p, p) == way


def test_tiles_only_where_they_fit(mx):
    # the rings want inner dimensions of more than three and five tiles of 128; a lane's offsets in D are 32 bits
    for n, least in ((384, DIRECT), (640, TILE)):
        assert mx._lib.ozimmu_mx_choose(8192, n, 8192, 8192) in (DIRECT, least)
    assert mx._lib.ozimmu_mx_choose(8192, 8192, 8192, 1 << 24) == DIRECT
    assert mx._lib.ozimmu_mx_choose(8192, 8192, 8192, (1 << 24) - 1) == TILE


def test_sizes_of_packed_matrices_and_workspaces(mx):
    assert mx.packed_bytes(1, 1) == 17408 and mx.packed_bytes(256, 128) == 17408 and mx.packed_bytes(257, 129) == 4 * 17408
    assert mx.packed_bytes(0, 5) == 0 and mx.packed_bytes(2 ** 22, 5) == 0 and mx.packed_bytes(5, 2 ** 29 + 1) == 0
    # few rows take one launch and no workspace; others hold X packed
    assert all(mx.workspace_bytes(m, n, p) == 0 for m in range(mx.FEW_ROWS + 1) for n in (1, 4096, 2 ** 20) for p in (1, 8192, 2 ** 21))
    assert mx.workspace_bytes(1, 4096, 4096) == 0 and mx.workspace_bytes(16, 8192, 2 ** 20) == 0
    assert mx.workspace_bytes(64, 4096, 4096) == 0 and mx.workspace_bytes(64, 4096, 8192) == mx.packed_bytes(64, 4096)
    assert mx.workspace_bytes(300, 512, 512) == mx.packed_bytes(300, 512)
    assert mx.backward_workspace_bytes(300, 512, 200) == mx.packed_bytes(300, 200) + mx.packed_bytes(200, 300) + mx.packed_bytes(512, 300)
