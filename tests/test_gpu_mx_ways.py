"""Every way of running a product of microscaled 4-bit matrices, forced where the library would choose another, against the product of
the same values in 64 bits (bounds as for the library's choice)."""
import numpy as np
import pytest

from oracle import mx as ref
from test_gpu_mx_product import EPS, TINY, TYPES, check, f64, matrix

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

# (rows, inner dimension, columns): one tile, several, edges in both directions, one to nine inner tiles and more, whole tiles only
SHAPES = [(1, 1, 1), (5, 129, 300), (256, 128, 256), (256, 512, 512), (257, 640, 255), (513, 300, 260), (300, 1100, 1037), (512, 1280, 768),
          (700, 2049, 515), (1024, 384, 1280), (2100, 257, 2300), (4352, 640, 4400)]


@pytest.fixture(scope="module")
def mx():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU: the HIP path has no CPU fallback")
    from paper_2409_13313_amd import mx
    return mx


def product(A, B):
    """A B^T in 64 bits (on the GPU where it is large), and the sum of magnitudes."""
    a, b = torch.from_numpy(A).cuda(), torch.from_numpy(B).cuda()
    return (a @ b.t()).cpu().numpy(), (a.abs() @ b.abs().t()).cpu().numpy()


@pytest.mark.parametrize("m,n,p", SHAPES)
@pytest.mark.parametrize("way", ["direct", "tile", "half"])
def test_way(mx, way, m, n, p):
    print(f"{way} {m} x {n} x {p}", flush=True)
    A, B = matrix(m, n, "bf16", m + n), matrix(p, n, "bf16", p + n + 1)
    qa, qb = ref.read_back(f64(A)), ref.read_back(f64(B))
    want, size = product(qa, qb)
    bound = max(n, 1) * 2.0 ** -23 * size
    (PA, _), (PB, _) = mx.quantize(A), mx.quantize(B)
    if n <= {"direct": 0, "tile": 384, "half": 640}[way]:     # (their rings have four and six places: inner dimensions that fill them)
        with pytest.raises(Exception, match="this way"):
            mx.gemm(PA, PB, way=way)
        return
    for kind, t in TYPES.items():
        check(mx.gemm(PA, PB, t, way=way), want, bound, kind, n, kind)
        big = torch.full((m + 1, p + 3), 5.0, dtype=t, device="cuda")
        mx.gemm(PA, PB, D=big[:m, 1:p + 1], way=way)
        check(big[:m, 1:p + 1], want, bound, kind, n, kind)
        assert (big[:, 0] == 5).all() and (big[:, p + 1:] == 5).all() and (big[m] == 5).all()
        old = matrix(m, p, kind, 3)
        got = mx.gemm(PA, PB, alpha=-0.5, beta=2.0, D=old.clone(), way=way)
        limit = 0.5 * bound + 3 * 2.0 ** -24 * (0.5 * (np.abs(want) + bound) + 2 * np.abs(f64(old)))
        check(got, -0.5 * want + 2.0 * f64(old), limit, kind, n, kind)


@pytest.mark.parametrize("way", ["direct", "tile", "half"])
def test_again_and_again(mx, way):
    """The same bits from call to call, with other work between."""
    m, n, p = 1800, 900, 2000
    (PA, _), (PB, _) = mx.quantize(matrix(m, n, "bf16", 1)), mx.quantize(matrix(p, n, "bf16", 2))
    first = mx.gemm(PA, PB, torch.bfloat16, way=way)
    for k in range(20):
        D = torch.full((m, p), float("nan"), dtype=torch.bfloat16, device="cuda")
        mx.gemm(PA, PB, D=D, way=way)
        assert torch.equal(D, first), k


# several tiles a workgroup, one behind the other: as many inner tiles as the ring has places, one more, several more; whole tiles, whose stores
# may be on their way in the next one's first stages, and edges
SEVERAL = [("tile", 4352, 512, 4096), ("tile", 4352, 513, 4100), ("tile", 4096, 1000, 4608), ("half", 4096, 700, 2560), ("half", 4096, 896, 2600),
           ("half", 4090, 1281, 2560)]


@pytest.mark.parametrize("way,m,n,p", SEVERAL)
def test_several_tiles_a_workgroup(mx, way, m, n, p):
    print(f"{way} {m} x {n} x {p}", flush=True)
    A, B = matrix(m, n, "bf16", m + n), matrix(p, n, "bf16", p + n + 1)
    want, size = product(ref.read_back(f64(A)), ref.read_back(f64(B)))
    (PA, _), (PB, _) = mx.quantize(A), mx.quantize(B)
    for kind in ("bf16", "f32"):
        check(mx.gemm(PA, PB, TYPES[kind], way=way), want, n * 2.0 ** -23 * size, kind, n, kind)


# results that are written past the caches: large gradients of weights (whole tiles and edges, both tile kernels), a product that with its
# operands is larger than the memory-side cache
@pytest.mark.parametrize("m,n,p,kind", [(1000, 2200, 2100, "f32"), (600, 2304, 4096, "f32"), (1000, 2304, 4096, "bf16"), (600, 4100, 2304, "f32")])
def test_large_gradient_of_weights(mx, m, n, p, kind):
    print(f"gradient of weights {m} x {n} x {p} {kind}", flush=True)
    X, G = matrix(m, n, "bf16", 1), matrix(m, p, "bf16", 2)
    want, size = product(ref.read_back(f64(G).T), ref.read_back(f64(X).T))
    dW = torch.full((p, n), float("nan"), dtype=TYPES[kind], device="cuda")
    mx.linear_backward(G, X, None, dW=dW)
    check(dW, want, m * 2.0 ** -23 * size, kind, m, "dW")


def test_product_larger_than_the_caches(mx):
    m, n, p = 8192, 512, 8192
    A, B = matrix(m, n, "bf16", 1), matrix(p, n, "bf16", 2)
    (PA, _), (PB, _) = mx.quantize(A), mx.quantize(B)
    whole = mx.gemm(PA, PB, torch.float32)
    rows = np.r_[0:40, 4090:4130, 8150:8192]
    a, b = torch.from_numpy(ref.read_back(f64(A)[rows])), torch.from_numpy(ref.read_back(f64(B)))
    want, size = (a @ b.t()).numpy(), (a.abs() @ b.abs().t()).numpy()
    check(whole[torch.from_numpy(rows).cuda()], want, n * 2.0 ** -23 * size, "f32", n)


# few rows, quantised on the way: every number of fragments a workgroup and of tiles at a time, more than one group of 16 rows
FEW = [(3, 700, 200), (10, 700, 200), (4, 1030, 5000), (13, 1030, 5000), (2, 1100, 9000), (12, 1100, 9000), (12, 900, 20000), (16, 2050, 16500),
       (40, 1500, 3000), (64, 33, 4000), (17, 4099, 64), (50, 129, 130)]


@pytest.mark.parametrize("m,n,p", FEW)
@pytest.mark.parametrize("kind", list(TYPES))
def test_few_rows(mx, m, n, p, kind):
    print(f"few {m} x {n} x {p} {kind}", flush=True)
    assert mx.workspace_bytes(m, n, p) == 0                 # (what takes one launch needs none)
    W = matrix(p, n, "bf16", p + n)
    PW, _ = mx.quantize(W)
    qw = ref.read_back(f64(W))
    for pad in (0, 1, 8):
        X = matrix(m, n, kind, m + n + pad, pad=pad)
        want, size = product(ref.read_back(f64(X)), qw)
        bound = n * 2.0 ** -23 * size
        for out in TYPES:
            check(mx.linear(X, PW, dtype=TYPES[out]), want, bound, out, n, f"{kind} to {out}, pad {pad}")


def test_gradient_of_a_large_layer(mx):
    """Each launch by itself, tiles of every size."""
    m, n, p = 4096, 2048, 2304
    X, W, G = matrix(m, n, "bf16", 1), matrix(p, n, "bf16", 2), matrix(m, p, "bf16", 3, std=1e-3)
    _, Wt = mx.quantize(W, rows=False, cols=True)
    dX, dW = mx.linear_backward(G, X, Wt)
    want, size = product(ref.read_back(f64(G)), ref.read_back(f64(W).T))
    check(dX, want, p * 2.0 ** -23 * size, "bf16", p, "dX")
    want, size = product(ref.read_back(f64(G).T), ref.read_back(f64(X).T))
    check(dW, want, m * 2.0 ** -23 * size, "f32", m, "dW")
