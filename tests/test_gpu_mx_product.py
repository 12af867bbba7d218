"""Products of microscaled 4-bit matrices, the linear layer and its gradient against products of the same quantised values in 64 bits.

Bounds: FP32 sums in any order are within n 2^-23 sum |a b| of the exact ones (the products of two 4-bit values and two powers of two
are exact); alpha and beta each add at most two FP32 roundings, and the result is rounded once to its type."""
import numpy as np
import pytest

from oracle import mx as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 2.0 ** -126, "bf16": 2.0 ** -126, "f16": 2.0 ** -24}
# one row and many, sizes around the tiles' edges, long inner dimensions with few outputs, an inner dimension of one
SHAPES = [(1, 1, 1), (1, 4096, 64), (1, 32, 4099), (2, 100, 33), (3, 129, 17), (15, 500, 250), (16, 1024, 1000), (17, 2050, 300), (33, 640, 129),
          (64, 64, 64), (65, 127, 255), (100, 8200, 70), (128, 256, 512), (133, 2051, 1283), (256, 384, 256), (257, 128, 300),
          (300, 5000, 257), (512, 1024, 513), (777, 1001, 513), (1100, 900, 1300)]


@pytest.fixture(scope="module")
def mx():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU: the HIP path has no CPU fallback")
    from paper_2409_13313_amd import mx
    return mx


def matrix(rows, n, kind, seed, pad=0, std=1.0):
    rng = np.random.default_rng(seed)
    x = std * rng.standard_normal((rows, n + pad)) * np.exp(0.5 * rng.standard_normal((rows, n + pad)))
    if rows > 3:
        x[rows // 2] = 0.0
    return torch.from_numpy(x).to(TYPES[kind]).cuda()[:, :n]


def f64(t):
    return t.double().cpu().numpy()


def check(got, want, bound, kind, n, what=""):
    got = f64(got)
    limit = bound + EPS[kind] * (np.abs(want) + bound) + TINY[kind]
    off = np.abs(got - want)
    assert (off <= limit).all(), f"{what}: {(off / np.maximum(limit, 1e-300)).max():.3g} of the bound at {np.unravel_index((off - limit).argmax(), off.shape)}"


@pytest.mark.parametrize("m,n,p", SHAPES)
def test_product(mx, m, n, p):
    print(f"product {m} x {n} x {p}", flush=True)
    A, B = matrix(m, n, "bf16", m + n), matrix(p, n, "bf16", p + n + 1)
    qa, qb = ref.read_back(f64(A)), ref.read_back(f64(B))
    want, bound = qa @ qb.T, ref.product_bound(qa, qb, n)
    (PA, _), (PB, _) = mx.quantize(A), mx.quantize(B)
    for kind, t in TYPES.items():
        check(mx.gemm(PA, PB, t), want, bound, kind, n, kind)
        # rows that begin anywhere; what lies around the output is left alone
        big = torch.full((m + 1, p + 3), 5.0, dtype=t, device="cuda")
        mx.gemm(PA, PB, D=big[:m, 1:p + 1])
        check(big[:m, 1:p + 1], want, bound, kind, n, kind)
        assert (big[:, 0] == 5).all() and (big[:, p + 1:] == 5).all() and (big[m] == 5).all()


@pytest.mark.parametrize("m,n,p", SHAPES)
@pytest.mark.parametrize("kind", list(TYPES))
def test_linear(mx, m, n, p, kind):
    print(f"linear {m} x {n} x {p} {kind}", flush=True)
    W = matrix(p, n, "f32", p + n)
    PW, _ = mx.quantize(W)
    qw = ref.read_back(f64(W))
    for pad in (0, 1):
        X = matrix(m, n, kind, m + n + 2, pad=pad)
        qx = ref.read_back(f64(X))
        Y = mx.linear(X, PW)
        assert Y.dtype is TYPES[kind]
        check(Y, qx @ qw.T, ref.product_bound(qx, qw, n), kind, n, f"pad {pad}")


@pytest.mark.parametrize("m,n,p", [(1, 300, 200), (20, 300, 70), (130, 200, 300), (300, 1100, 520)])
@pytest.mark.parametrize("alpha,beta", [(1.0, 1.0), (-0.5, 0.0), (2.0, -0.25), (0.0, 1.0)])
def test_alpha_and_beta(mx, m, n, p, alpha, beta):
    X, W = matrix(m, n, "bf16", 1), matrix(p, n, "bf16", 2)
    PX, PW = mx.quantize(X)[0], mx.quantize(W)[0]
    qx, qw = ref.read_back(f64(X)), ref.read_back(f64(W))
    product, bound = qx @ qw.T, ref.product_bound(qx, qw, n)
    for kind, t in TYPES.items():
        old = matrix(m, p, kind, 3)
        if beta == 0.0:
            old[:, ::3] = float("nan")          # not read
        want = alpha * product + (beta * f64(old) if beta else 0.0)
        # alpha s, beta c and their sum: three FP32 roundings
        limit = abs(alpha) * bound + 3 * 2.0 ** -24 * (abs(alpha) * (np.abs(product) + bound) + (abs(beta * f64(old)) if beta else 0.0))
        for D in (mx.gemm(PX, PW, alpha=alpha, beta=beta, D=old.clone()), mx.linear(X, PW, alpha=alpha, beta=beta, D=old.clone())):
            check(D, want, limit, kind, n, kind)


@pytest.mark.parametrize("m,n,p", [(1, 64, 32), (8, 100, 60), (33, 70, 129), (200, 520, 300), (777, 1001, 513)])
@pytest.mark.parametrize("kind", list(TYPES))
def test_gradient(mx, m, n, p, kind):
    print(f"gradient {m} x {n} x {p} {kind}", flush=True)
    X, W, G = matrix(m, n, kind, 1, pad=1), matrix(p, n, kind, 2), matrix(m, p, kind, 3, pad=3)
    _, Wt = mx.quantize(W, rows=False, cols=True)
    dX, dW = mx.linear_backward(G, X, Wt)
    assert dX.dtype is TYPES[kind] and dW.dtype is torch.float32
    qg, qwt = ref.read_back(f64(G)), ref.read_back(f64(W).T)
    qgt, qxt = ref.read_back(f64(G).T), ref.read_back(f64(X).T)
    check(dX, qg @ qwt.T, ref.product_bound(qg, qwt, p), kind, p, "dX")
    check(dW, qgt @ qxt.T, ref.product_bound(qgt, qxt, m), "f32", m, "dW")
    # one of them alone, and added to what is there
    only, none = mx.linear_backward(G, None, Wt)
    assert none is None and torch.equal(only, dX)
    none, only = mx.linear_backward(G, X, None)
    assert none is None and torch.equal(only, dW)
    twice = mx.linear_backward(G, X, Wt, beta_w=1.0, dW=dW.clone())[1]
    check(twice, 2 * (qgt @ qxt.T), 2 * ref.product_bound(qgt, qxt, m) + 2.0 ** -22 * np.abs(f64(dW)), "f32", m, "dW twice")


def test_gradient_against_differences(mx):
    """On values that the form holds exactly in both directions quantisation changes nothing, the layer is linear in each operand, and
    differences of sum(G Y) are its gradient up to the rounding of Y."""
    rng = np.random.default_rng(4)
    m, n, p = 40, 96, 64
    grid = np.array([-6, -4, -3, -2, -1.5, -1, -0.5, 0, 0.5, 1, 1.5, 2, 3, 4, 6])

    def held(rows, cols):
        x = rng.choice(grid, (rows, cols))
        x[::8, :] = rng.choice([-4.0, 4.0, 6.0], x[::8, :].shape)   # every block of 32, either way, has the scale 2^0
        x[:, ::8] = rng.choice([-4.0, 4.0, 6.0], x[:, ::8].shape)
        return x

    X, W, G = held(m, n), held(p, n), held(m, p)
    dev = lambda a: torch.from_numpy(a).float().cuda()  # noqa: E731
    loss = lambda x, w: float((f64(mx.linear(dev(x), mx.quantize(dev(w))[0])) * G).sum())  # noqa: E731
    dX, dW = mx.linear_backward(dev(G), dev(X), mx.quantize(dev(W), rows=False, cols=True)[1])
    base = loss(X, W)
    for _ in range(24):
        # a step from one held value to another: sums of multiples of 1/4 below 2^24 / 4 are exact in FP32, and so is the difference
        i, l, j = rng.integers(m), rng.integers(n), rng.integers(p)
        if i % 8 and l % 8:
            X2 = X.copy()
            X2[i, l] = rng.choice(grid)
            assert loss(X2, W) - base == (X2[i, l] - X[i, l]) * float(dX[i, l])
        if j % 8 and l % 8:
            W2 = W.copy()
            W2[j, l] = rng.choice(grid)
            assert loss(X, W2) - base == (W2[j, l] - W[j, l]) * float(dW[j, l])


@pytest.mark.parametrize("m", [1, 5, 64, 300])
def test_what_is_not_finite_stays_in_its_rows(mx, m):
    n, p = 300, 200
    X, W = matrix(m, n, "bf16", 1), matrix(p, n, "bf16", 2)
    X[m // 2, 77], W[150, 200] = float("inf"), float("nan")
    Y = f64(mx.linear(X, mx.quantize(W)[0]))
    bad = np.zeros((m, p), dtype=bool)
    bad[m // 2, :] = bad[:, 150] = True
    assert np.array_equal(np.isnan(Y), bad)


def test_scales_at_both_ends(mx):
    """Blocks with the largest and the least scale: products from overflow to nothing."""
    n = 128
    X = torch.zeros((4, n), device="cuda")
    X[0], X[1], X[2], X[3] = 2.0 ** 125, 2.0 ** -126, 1.0, 0.0
    W = torch.zeros((3, n), device="cuda")
    W[0], W[1], W[2] = 2.0 ** -125, 1.0, 2.0 ** 10
    got = f64(mx.linear(X, mx.quantize(W)[0]))
    with np.errstate(over="ignore"):
        want = (f64(X) @ f64(W).T).astype(np.float32).astype(np.float64)
    assert np.array_equal(got[:, 0], want[:, 0]) or np.allclose(got[:, 0], want[:, 0], rtol=0, atol=n * 2.0 ** -126)
    assert np.allclose(got[:, 1:], want[:, 1:], rtol=2.0 ** -20, atol=n * 2.0 ** -126)


def test_nothing_to_sum_or_to_write(mx):
    for m, n, p in ((0, 64, 8), (8, 64, 0), (4, 0, 6)):
        X = torch.ones((m, n), device="cuda")
        W = mx.quantize(torch.ones((p, n), device="cuda"))[0]
        Y = mx.linear(X, W)
        assert Y.shape == (m, p) and (Y == 0).all()
        D = torch.ones((m, p), device="cuda")
        mx.linear(X, W, beta=0.5, D=D)
        assert (D == 0.5).all() if n == 0 else True
    G, X = torch.ones((0, 8), device="cuda"), torch.ones((0, 40), device="cuda")
    dX, dW = mx.linear_backward(G, X, mx.quantize(torch.ones((8, 40), device="cuda"), rows=False, cols=True)[1])
    assert dX.shape == (0, 40) and dW.shape == (8, 40) and (dW == 0).all()


def test_same_bits_again_on_another_stream_and_in_a_graph(mx):
    m, n, p = 200, 3000, 400
    X, W, G = matrix(m, n, "bf16", 1), matrix(p, n, "bf16", 2), matrix(m, p, "bf16", 3)
    by_row, by_col = mx.quantize(W, rows=True, cols=True)
    ws, bws = mx.alloc_workspace(m, n, p), mx.alloc_workspace(m, n, p, backward=True)
    Y, dX, dW = (torch.empty(s, dtype=torch.float32, device="cuda") for s in ((m, p), (m, n), (p, n)))

    def step():
        mx.linear(X, by_row, D=Y, workspace=ws)
        mx.linear_backward(G, X, by_col, dX=dX, dW=dW, workspace=bws)

    step()
    want = [t.clone() for t in (Y, dX, dW)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(a, b) for a, b in zip(want, (Y, dX, dW)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    X2 = matrix(m, n, "bf16", 9)
    for x in (X.clone(), X2, X.clone()):
        X.copy_(x)
        for t in (Y, dX, dW):
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in (Y, dX, dW)]
        step()
        assert all(torch.equal(a, b) for a, b in zip(replayed, (Y, dX, dW)))
