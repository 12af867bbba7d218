"""The gradient of the weights where the gradients of the losses are orders of magnitude apart, against the definition in 64 bits.

What a token gives to dW is its slopes times g x.  Bounds: slopes and logits as in test_gpu_lm_loss.py.  In BF16 x g / max|g| is rounded by half a step, 2^-8.  In FP16
it is held times a power of two: 2^-11 of itself, or 2^-21 of the largest |x| of its row, or, where it is not made smaller than x, half of x's own least
step, 2^-25; then one more rounding of dW where tokens are added afterwards."""
import pytest

torch = pytest.importorskip("torch")
from test_gpu_lm_loss import HALF, IGNORE, TYPES, exact, lm  # noqa: E402,F401

pytestmark = pytest.mark.gpu


def check_rows(dW, X, d, g, size, kind, out, what, beta=0.0, old=None):
    """dW element by element (d: slopes without g, in 64 bits)."""
    x = X.double()
    gd = d * g.unsqueeze(1)
    p = (d + (d < 0)).abs()
    off_d = (HALF[kind] * d.abs() + 2.0 ** -40 + (size.unsqueeze(1) * 2 + 2.0 ** -20) * p) * g.abs().unsqueeze(1)
    least = torch.clamp(2.0 ** -21 * x.abs().amax(1, keepdim=True), min=2.0 ** -25) if kind == "f16" else torch.zeros_like(x[:, :1])
    want = gd.t() @ x
    # (2^-18: sums of fewer than 1000 terms in FP32, roundings of 2^-23)
    bound = off_d.t() @ x.abs() + (HALF[kind] + 2.0 ** -18) * (gd.abs().t() @ x.abs()) + gd.abs().t() @ least.expand_as(x)
    if beta:
        want = want + beta * old.double()
        bound = bound + 2.0 ** -22 * beta * old.double().abs()
    off = (dW.double() - want).abs()
    limit = bound + 2 * HALF[out] * (want.abs() + bound) + {"f16": 2.0 ** -24}.get(out, 1e-38)
    assert (off <= limit).all(), f"{what}: {(off / limit).max().item():.3g} of the bound"
    return want, limit


def parted(m, n, p, kind, pad, seed, magnitudes):
    """Tokens in as many classes as there are magnitudes of g; a class has words of its own, which the others do not give anything (their logits lie 65504 lower: zero
    probability in 64 bits as well)."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    classes = len(magnitudes)
    X = torch.randn((m, n + pad), device="cuda", generator=gen)
    W = torch.randn((p, n + pad), device="cuda", generator=gen) * n ** -0.5
    token, word = torch.arange(m, device="cuda") % classes, torch.arange(p, device="cuda") % classes
    for c in range(classes):
        X[:, c], W[:, c] = (token == c).float(), torch.where(word == c, 0.0, -65504.0)
    y = torch.randint(0, p // classes, (m,), device="cuda", generator=gen) * classes + token
    g = (torch.rand(m, device="cuda", generator=gen) + 0.5) * torch.tensor(magnitudes, device="cuda")[token]
    g = torch.where(torch.rand(m, device="cuda", generator=gen) < 0.5, g, -g)
    y[m // 2] = IGNORE
    return X.to(TYPES[kind])[:, :n], W.to(TYPES[kind])[:, :n], y, g, word


@pytest.mark.parametrize("m,n,p,pad", [(6, 64, 60, 0), (90, 136, 500, 0), (90, 131, 500, 1), (300, 264, 1000, 0)])
@pytest.mark.parametrize("magnitudes", [(1.0, 1e-8), (1.0, 1e-5, 1e-7, 1e-30), (1e-20, 1e-3, 30.0), (3e-36, 1e-37)])
@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_words_of_tokens_whose_gradient_is_small(lm, m, n, p, pad, magnitudes, kind):  # noqa: F811
    X, W, y, g, word = parted(m, n, p, kind, pad, m + n, magnitudes)
    loss, lse = lm.cross_entropy(X, W, y)
    _, _, size, d = exact(X, W, y, g)
    part = (X.double().abs() @ W.double().abs().t()) * (6 * n / 32 + 8) * 2.0 ** -23
    size = torch.where(part > 100 * (6 * n / 32 + 8) * 2.0 ** -23 * n, 0.0, part).amax(1)   # (of the words that have a part in the sum)
    for out in ("f32", kind):
        dX, dW = lm.cross_entropy_backward(g, X, W, y, lse, dw_type=TYPES[out])
        want, limit = check_rows(dW, X, d, g.double(), size, kind, out, f"{kind} {out}")
        if out == "f32":
            # each class's rows of dW, as a whole, are there to the digits of their own
            for c, magnitude in enumerate(magnitudes):
                rows = word == c
                assert (dW[rows].double() - want[rows]).norm() <= 4 * HALF[kind] * want[rows].norm(), (c, magnitude)
        again = lm.cross_entropy_backward(g, X, W, y, lse, dw_type=TYPES[out])
        assert torch.equal(again[0], dX) and torch.equal(again[1], dW)
    old = torch.randn((p, n), device="cuda") * max(magnitudes)
    got = old.clone()
    lm.cross_entropy_backward(g, X, W, y, lse, dW=got, beta=0.5, need_dx=False)
    check_rows(got, X, d, g.double(), size, kind, "f32", "beta", 0.5, old)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_states_of_every_magnitude(lm, kind):  # noqa: F811
    """Rows of X from the least to the largest numbers, g all the same: nothing is rounded that would not be by itself."""
    m, n, p = 60, 72, 200
    gen = torch.Generator(device="cuda").manual_seed(3)
    X = torch.randn((m, n), device="cuda", generator=gen) * 2.0 ** torch.linspace(-20, 13, m, device="cuda").unsqueeze(1)
    W = torch.randn((p, n), device="cuda", generator=gen) * n ** -0.5 * 2.0 ** -13
    X, W = X.to(TYPES[kind]), W.to(TYPES[kind])
    y = torch.randint(0, p, (m,), device="cuda", generator=gen)
    for g in (torch.full((m,), 1 / 60, device="cuda"), 2.0 ** torch.linspace(0, -40, m, device="cuda"), 2.0 ** torch.linspace(-40, 0, m, device="cuda")):
        _, lse = lm.cross_entropy(X, W, y)
        _, _, size, d = exact(X, W, y, g)
        _, dW = lm.cross_entropy_backward(g, X, W, y, lse, dw_type=torch.float32)
        check_rows(dW, X, d, g.double(), size, kind, "f32", kind)


def test_a_vocabulary_in_pieces(lm):  # noqa: F811
    """Slopes of 131072 words at a time for 300 tokens; every eighth token's g is far below the others'."""
    m, n, p = 300, 40, 270001
    gen = torch.Generator(device="cuda").manual_seed(8)
    X = torch.randn((m, n), device="cuda", generator=gen)
    W = torch.randn((p, n), device="cuda", generator=gen) * n ** -0.5
    far = torch.arange(m, device="cuda") % 8 == 3
    words = torch.arange(p, device="cuda") % 5 == 1
    X[:, 0], X[:, 1] = far.float(), (~far).float()
    W[:, 0], W[:, 1] = torch.where(words, 0.0, -65504.0), torch.where(words, -65504.0, 0.0)
    X, W = X.half(), W.half()
    y = torch.randint(0, p // 5 - 1, (m,), device="cuda", generator=gen) * 5 + far.long()
    g = torch.where(far, 1e-9, 1.0) * (torch.rand(m, device="cuda", generator=gen) + 0.5)
    _, lse = lm.cross_entropy(X, W, y)
    _, _, _, d = exact(X, W, y, g)
    size = torch.full((m,), 6 * n * (6 * n / 32 + 8) * 2.0 ** -23, device="cuda", dtype=torch.float64)   # (|x| below 6, |w| below 1 in words with a part)
    dX, dW = lm.cross_entropy_backward(g, X, W, y, lse, dw_type=torch.float32)
    want, _ = check_rows(dW, X, d, g.double(), size, "f16", "f32", "pieces")
    assert (dW[words].double() - want[words]).norm() <= 4 * HALF["f16"] * want[words].norm()


def test_a_captured_gradient_with_other_tokens_far(lm):  # noqa: F811
    """Captured where no token's g is far below the others', replayed where many are, and back: which they are is found at each replay."""
    X, W, y, g, _ = parted(90, 136, 500, "f16", 0, 3, (1.0, 1e-7, 1e-30))
    even = torch.sign(g)
    _, lse = lm.cross_entropy(X, W, y)
    held = even.clone()
    room = torch.empty(lm.cross_entropy_workspace_bytes(90, 136, 500, True), dtype=torch.uint8, device="cuda")
    dX, dW = torch.empty_like(X), torch.empty((500, 136), device="cuda")
    run = lambda: lm.cross_entropy_backward(held, X, W, y, lse, dX=dX, dW=dW, workspace=room)  # noqa: E731
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for i in range(5):
        now = g if i % 2 == 0 else even
        held.copy_(now)
        room.fill_(255)
        graph.replay()
        want = lm.cross_entropy_backward(now, X, W, y, lse, dw_type=torch.float32)      # (eager work between replays)
        assert torch.equal(dX, want[0]) and torch.equal(dW, want[1]), i
        if i % 3 == 0:
            torch.cuda.synchronize()


def test_gradients_that_are_not_finite(lm):  # noqa: F811
    """A g that is a NaN or an infinity, or a row of X that holds one: what comes of it is no number in the rows and words that it reaches, and those are
    dX's row of that token and all of dW."""
    X, W, y, g, _ = parted(30, 64, 60, "f16", 0, 4, (1.0, 1e-9))
    _, lse = lm.cross_entropy(X, W, y)
    want = lm.cross_entropy_backward(g, X, W, y, lse)[0]
    for row in (0, 1):                                                # (of either magnitude)
        for bad in (float("nan"), float("inf")):
            h = g.clone()
            h[row] = bad
            dX, dW = lm.cross_entropy_backward(h, X, W, y, lse, dw_type=torch.float32)
            rest = torch.arange(30, device="cuda") != row
            assert torch.equal(dX[rest], want[rest]) and not torch.isfinite(dX[row]).any() and not torch.isfinite(dW[y[row]]).any()
            V = X.clone()
            V[row, 5] = bad
            _, other = lm.cross_entropy(V, W, y)
            dX, dW = lm.cross_entropy_backward(g, V, W, y, other, dw_type=torch.float32)
            assert torch.equal(dX[rest], want[rest]) and not torch.isfinite(dW).any()
