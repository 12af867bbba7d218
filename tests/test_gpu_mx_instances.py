"""Shapes that run an instance of the direct kernels (csrc/ozimmu_mx_gemm.hip) which no other shape of these tests does: two fragments of B a
workgroup beside eight waves, and two products in one launch of which one has a long inner dimension.  Products of the same quantised values
in 64 bits, bounds as for the other products."""
import pytest

from oracle import mx as ref
from test_gpu_mx_product import TYPES, check, f64, matrix, mx  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DIRECT = 0


# 65 to 128 units of 64 x 64 outputs and 32 inner tiles or more: k_mx_direct<2, 8>
@pytest.mark.parametrize("m,n,p", [(256, 4096, 2048), (250, 4101, 1990), (65, 4000, 4093)])
@pytest.mark.parametrize("kind", list(TYPES))
def test_two_fragments_eight_waves(mx, m, n, p, kind):  # noqa: F811
    print(f"product {m} x {n} x {p} {kind}", flush=True)
    units, tiles = -(-m // 64) * -(-p // 64), -(-n // 128)
    assert 64 < units <= 128 and tiles >= 32 and mx._lib.ozimmu_mx_choose(m, n, p, p) == DIRECT
    X, W = matrix(m, n, kind, m + n, pad=1), matrix(p, n, kind, p + n + 1)
    qx, qw = ref.read_back(f64(X)), ref.read_back(f64(W))
    want, bound = qx @ qw.T, ref.product_bound(qx, qw, n)
    PX, PW = mx.quantize(X)[0], mx.quantize(W)[0]
    big = torch.full((m + 1, p + 3), 5.0, dtype=TYPES[kind], device="cuda")
    mx.gemm(PX, PW, D=big[:m, 1:p + 1])
    check(big[:m, 1:p + 1], want, bound, kind, n, "product")
    assert (big[:, 0] == 5).all() and (big[:, p + 1:] == 5).all() and (big[m] == 5).all()
    check(mx.linear(X, PW), want, bound, kind, n, "linear")


# both gradients in one launch, one of them over a long inner dimension or both: k_mx_direct2<2, 8> (65 units, the long one second and first, and
# 126, both), <1, 8> (64 units, the long one second and first), <2, 4> (130 units, both)
@pytest.mark.parametrize("m,n,p,units", [(4096, 64, 64, 65), (64, 64, 4096, 65), (4090, 63, 60, 65), (4000, 64, 64, 64), (64, 64, 4032, 64),
                                         (4097, 32, 4128, 130), (4000, 33, 4001, 126)])
@pytest.mark.parametrize("kind", list(TYPES))
def test_two_products_of_which_one_is_long(mx, m, n, p, units, kind):  # noqa: F811
    print(f"gradient {m} x {n} x {p} {kind}", flush=True)
    tiles = lambda k: -(-k // 64)  # noqa: E731
    assert tiles(m) * tiles(n) + tiles(p) * tiles(n) == units and max(m, p) > 31 * 128
    assert mx._lib.ozimmu_mx_choose(m, p, n, n) == DIRECT and mx._lib.ozimmu_mx_choose(p, m, n, n) == DIRECT
    X, W, G = matrix(m, n, kind, 1, pad=1), matrix(p, n, kind, 2), matrix(m, p, kind, 3, pad=3)
    _, Wt = mx.quantize(W, rows=False, cols=True)
    dX, dW = mx.linear_backward(G, X, Wt)
    qg, qwt = ref.read_back(f64(G)), ref.read_back(f64(W).T)
    qgt, qxt = ref.read_back(f64(G).T), ref.read_back(f64(X).T)
    check(dX, qg @ qwt.T, ref.product_bound(qg, qwt, p), kind, p, "dX")
    check(dW, qgt @ qxt.T, ref.product_bound(qgt, qxt, m), "f32", m, "dW")
