"""Packed matrices whose memory held NaN scales and largest codes before (0xff everywhere): rows that fill up a tile are not written, are multiplied
as they are, and may reach nothing that is stored.  And values that are not finite reach their row and their column alone, in every way
that a product can be run."""
import numpy as np
import pytest

from oracle import mx as ref
from test_gpu_mx_product import check, f64, matrix, mx  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
KINDS = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
# one tile and a row, several with edges both ways, several a workgroup; inner dimensions that end inside a block and a tile
SHAPES = [(257, 1100, 300), (130, 1000, 129), (700, 900, 521), (4353, 700, 4097)]


def poisoned(nbytes):
    return torch.full((nbytes,), 255, dtype=torch.uint8, device="cuda")


def quantized(mx, X, cols=False):  # noqa: F811
    """X quantised into memory full of 0xff, along its rows or its columns."""
    rows, n = X.shape
    P = mx.Packed(poisoned(mx.packed_bytes(*((n, rows) if cols else (rows, n)))), *((n, rows) if cols else (rows, n)))
    at = P.data.data_ptr()
    mx._check(mx._lib.ozimmu_mx_quantize(KINDS[X.dtype], rows, n, X.data_ptr(), X.stride(0), None if cols else at, at if cols else None,
                                         torch.cuda.current_stream().cuda_stream))
    return P


@pytest.mark.parametrize("m,n,p", SHAPES)
@pytest.mark.parametrize("way", ["direct", "tile", "half"])
def test_what_the_memory_held(mx, way, m, n, p):  # noqa: F811
    print(f"{way} {m} x {n} x {p}", flush=True)
    A, B = matrix(m, n, "bf16", 1), matrix(p, n, "bf16", 2)
    PA, PB = quantized(mx, A), quantized(mx, B)
    qa, qb = torch.from_numpy(ref.read_back(f64(A))).cuda(), torch.from_numpy(ref.read_back(f64(B))).cuda()
    want, size = (qa @ qb.t()).cpu().numpy(), (qa.abs() @ qb.abs().t()).cpu().numpy()
    for kind, t in (("f32", torch.float32), ("bf16", torch.bfloat16)):
        check(mx.gemm(PA, PB, t, way=way), want, n * 2.0 ** -23 * size, kind, n, kind)
        big = torch.full((m + 1, p + 3), 5.0, dtype=t, device="cuda")
        mx.gemm(PA, PB, D=big[:m, 1:p + 1], way=way)
        check(big[:m, 1:p + 1], want, n * 2.0 ** -23 * size, kind, n, kind)
        assert (big[:, 0] == 5).all() and (big[:, p + 1:] == 5).all() and (big[m] == 5).all()


@pytest.mark.parametrize("m,n,p", SHAPES)
@pytest.mark.parametrize("way", ["direct", "tile", "half"])
def test_what_is_not_finite(mx, way, m, n, p):  # noqa: F811
    print(f"{way} {m} x {n} x {p}", flush=True)
    A, B = matrix(m, n, "bf16", 1), matrix(p, n, "bf16", 2)
    rows, cols = [3, m - 1], [0, p - 2]
    A[rows[0], 77], A[rows[1], n - 1] = float("inf"), float("nan")
    B[cols[0], n - 1], B[cols[1], 200] = float("nan"), float("-inf")
    bad = np.zeros((m, p), dtype=bool)
    bad[rows, :] = bad[:, cols] = True
    PA, PB = quantized(mx, A), quantized(mx, B)
    finite = mx.gemm(quantized(mx, torch.nan_to_num(A, 0, 0, 0)), quantized(mx, torch.nan_to_num(B, 0, 0, 0)), way=way).cpu().numpy()
    for t in (torch.float32, torch.bfloat16):
        got = f64(mx.gemm(PA, PB, t, way=way))
        assert np.array_equal(np.isnan(got), bad), t
        if t is torch.float32:
            assert np.array_equal(got[~bad], finite[~bad].astype(np.float64))
        old = torch.ones((m, p), dtype=t, device="cuda")
        assert np.array_equal(np.isnan(f64(mx.gemm(PA, PB, beta=0.5, D=old, way=way))), bad), t


# few rows, quantised on the way, and more, quantised into a workspace
@pytest.mark.parametrize("m,n,p", [(1, 300, 200), (13, 1100, 300), (50, 129, 130), (100, 700, 300), (300, 1100, 521)])
def test_layer_and_gradient(mx, m, n, p):  # noqa: F811
    print(f"layer {m} x {n} x {p}", flush=True)
    X, W, G = matrix(m, n, "bf16", 1), matrix(p, n, "bf16", 2), matrix(m, p, "bf16", 3)
    by_row, by_col = quantized(mx, W), quantized(mx, W, cols=True)
    room = lambda: poisoned(mx.alloc_workspace(m, n, p, backward=True).numel())  # noqa: E731
    Y = mx.linear(X, by_row, workspace=room())
    dX, dW = mx.linear_backward(G, X, by_col, workspace=room())
    q = {k: ref.read_back(v) for k, v in (("x", f64(X)), ("w", f64(W)), ("g", f64(G)), ("xt", f64(X).T), ("wt", f64(W).T), ("gt", f64(G).T))}
    for got, a, b, inner, kind in ((Y, "x", "w", n, "bf16"), (dX, "g", "wt", p, "bf16"), (dW, "gt", "xt", m, "f32")):
        check(got, q[a] @ q[b].T, ref.product_bound(q[a], q[b], inner), kind, inner, a + b)
    X[m // 2, n - 1] = float("nan")
    bad = np.zeros((m, p), dtype=bool)
    bad[m // 2] = True
    assert np.array_equal(np.isnan(f64(mx.linear(X, by_row, workspace=room()))), bad)
    dX, dW = mx.linear_backward(G, X, by_col, workspace=room())
    bad = np.zeros((p, n), dtype=bool)
    bad[:, n - 1] = True
    assert np.array_equal(np.isnan(f64(dW)), bad) and not torch.isnan(dX).any()


def test_reading_back(mx):  # noqa: F811
    X = matrix(130, 300, "bf16", 4)
    for cols in (False, True):
        P, want = quantized(mx, X, cols), ref.read_back(f64(X).T if cols else f64(X))
        assert np.array_equal(f64(mx.dequantize(P)), want)
        codes, scales = mx.unpack(P)
        assert np.array_equal(f64(mx.dequantize(mx.pack(codes, scales, P.n))), want)
