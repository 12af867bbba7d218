"""Cross entropy of a linear layer's outputs and its gradient against the definition in 64 bits.

Bounds.  A logit is an FP32 sum of exact products: off by at most (6 n / 32 + 8) roundings of 2^-23 of sum |x w|.  The logarithm of the sum of exponentials is
off by no more than its logits and by 40 roundings of its own magnitude and of 1.  Slopes p - [v = y] are rounded to 16 bits (half a step each) and
the logits' error e changes them by e p; their products are FP32 sums, and results are rounded to their type."""
import numpy as np
import pytest

from oracle import lm as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
IGNORE = -100
# tokens, elements, words: one of each, sizes around fragments and tiles, rows that begin anywhere, each of the ways that a loss can go
SHAPES = [(1, 1, 1), (1, 8, 300), (1, 1024, 5000), (2, 33, 17), (5, 72, 129), (16, 64, 64), (17, 1001, 700), (40, 128, 2000), (64, 520, 4100), (65, 2048, 256),
          (130, 136, 5003), (257, 200, 129), (300, 1000, 3000), (520, 2048, 1111), (1000, 1001, 2050), (4100, 264, 4000)]


@pytest.fixture(scope="module")
def lm():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU: the HIP path has no CPU fallback")
    from paper_2409_13313_amd import lm
    return lm


def layer(m, n, p, kind, seed, pad=0, ignored=0.1, known=8.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    W = (torch.randn((p, n + pad), device="cuda", generator=gen) * n ** -0.5).to(TYPES[kind])[:, :n]
    y = torch.randint(0, p, (m,), device="cuda", generator=gen)
    X = torch.randn((m, n + pad), device="cuda", generator=gen)
    X[:, :n] += W[y].float() * torch.rand((m, 1), device="cuda", generator=gen) * known
    if m > 2:
        y[torch.rand(m, device="cuda", generator=gen) < ignored] = IGNORE
    return X.to(TYPES[kind])[:, :n], W, y


def exact(X, W, y, g=None, ignore=IGNORE):
    """On the GPU in 64 bits: loss, lse, slopes (without g), dX, dW and what their errors are bounded by."""
    x, w = X.double(), W.double()
    z = x @ w.t()
    lse = torch.logsumexp(z, 1)
    learnt = y != ignore
    at = torch.where(learnt, y, 0).unsqueeze(1)
    loss = torch.where(learnt, lse - z.gather(1, at).squeeze(1), 0.0)
    size = ((x.abs() @ w.abs().t()).amax(1) * (6 * X.shape[1] / 32 + 8) * 2.0 ** -23)
    if g is None:
        return loss, lse, size
    d = (z - lse.unsqueeze(1)).exp()
    d.scatter_add_(1, at, torch.full_like(loss, -1.0).unsqueeze(1))
    d = torch.where(learnt.unsqueeze(1), d, 0.0)
    return loss, lse, size, d


@pytest.mark.parametrize("m,n,p", SHAPES)
@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_loss(lm, m, n, p, kind):
    for pad in (0, 1, 8):
        print(f"loss {m} x {n} x {p} {kind} pad {pad}", flush=True)
        X, W, y = layer(m, n, p, kind, m + n + p, pad)
        loss, lse = lm.cross_entropy(X, W, y)
        want, want_lse, size = exact(X, W, y)
        limit = 2 * size + 40 * 2.0 ** -24 * (1 + want_lse.abs())
        assert ((lse.double() - want_lse).abs() <= limit).all() and ((loss.double() - want).abs() <= limit).all()
        assert (loss[y == IGNORE] == 0).all()
        again = lm.cross_entropy(X, W, y)
        assert torch.equal(again[0], loss) and torch.equal(again[1], lse)


def test_loss_of_a_word_that_has_nearly_all_keeps_its_digits(lm):
    X = torch.zeros((3, 64), device="cuda", dtype=torch.bfloat16)
    W = torch.zeros((1000, 64), device="cuda", dtype=torch.bfloat16)
    X[:, 0], W[7, 0] = torch.tensor([20.0, 30.0, 40.0], device="cuda").bfloat16(), 1.0
    y = torch.full((3,), 7, device="cuda")
    loss, _ = lm.cross_entropy(X, W, y)
    want = torch.log1p(999 * torch.exp(-X[:, 0].double()))
    assert ((loss.double() - want).abs() <= 1e-5 * want).all()


def test_oracle_and_this_files_formulas(lm):
    X, W, y = layer(20, 30, 40, "f16", 3)
    g = torch.randn(20, device="cuda")
    loss, lse, _, d = exact(X, W, y, g)
    a = (X.double().cpu().numpy(), W.double().cpu().numpy(), y.cpu().numpy())
    want = ref.cross_entropy(*a, IGNORE)
    assert np.allclose(loss.cpu().numpy(), want[0], atol=1e-13) and np.allclose(lse.cpu().numpy(), want[1], atol=1e-13)
    assert np.allclose((d * g.double().unsqueeze(1)).cpu().numpy(), ref.slopes(*a, g.double().cpu().numpy(), IGNORE), atol=1e-13)


def check_gradient(got, d, other, g, size, kind, out, along_tokens, what):
    """got against (g d) other (dX) or (g d)^T other (dW)."""
    gd = d * g.unsqueeze(1)
    p = (d + (d < 0)).abs()                                          # (about the probabilities)
    off_d = (HALF[kind] * d.abs() + 2.0 ** -40 + (size.unsqueeze(1) * 2 + 2.0 ** -20) * p) * g.abs().unsqueeze(1)
    if along_tokens:                                                 # X is rounded once more, times its row's share of the largest g
        want, bound = gd.t() @ other, (off_d.t() + (HALF[kind] + 2.0 ** -18) * gd.abs().t()) @ other.abs()
    else:
        want, bound = gd @ other, (off_d + 2.0 ** -18 * gd.abs()) @ other.abs()
    off = (got.double() - want).abs()
    limit = bound + HALF[out] * (want.abs() + bound) + {"f16": 2.0 ** -24}.get(out, 1e-38)
    assert (off <= limit).all(), f"{what}: {(off / limit).max().item():.3g} of the bound"
    return want


@pytest.mark.parametrize("m,n,p", SHAPES)
@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_gradient(lm, m, n, p, kind):
    for pad, dw_type in ((0, "f32"), (1, kind), (8, kind)):
        print(f"gradient {m} x {n} x {p} {kind} pad {pad}", flush=True)
        X, W, y = layer(m, n, p, kind, m + n + p, pad)
        gen = torch.Generator(device="cuda").manual_seed(m)
        for g in (torch.ones(m, device="cuda") / m, torch.randn(m, device="cuda", generator=gen)):
            _, lse = lm.cross_entropy(X, W, y)
            dX, dW = lm.cross_entropy_backward(g, X, W, y, lse, dw_type=TYPES[dw_type])
            _, _, size, d = exact(X, W, y, g)
            check_gradient(dX, d, W.double(), g.double(), size, kind, kind, False, "dX")
            check_gradient(dW, d, X.double(), g.double(), size, kind, dw_type, True, "dW")
            assert (dX[y == IGNORE] == 0).all()
            # one alone is the same, and the same call gives the same bits
            assert torch.equal(lm.cross_entropy_backward(g, X, W, y, lse, need_dw=False)[0], dX)
            assert torch.equal(lm.cross_entropy_backward(g, X, W, y, lse, dw_type=TYPES[dw_type], need_dx=False)[1], dW)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_gradient_against_differences_of_the_loss(lm, kind):
    """Along directions of +-1 in X: values are multiples of 2^-3 below 4, steps of 2^-5 (7 bits together).  With |W's columns| summed at about 2.5 a
    logit moves by 0.08, so the central difference is off by less than a hundredth (h^2 f''' / 6, with derivatives of about 1)."""
    m, n, p, h = 50, 40, 300, 2.0 ** -5
    gen = torch.Generator(device="cuda").manual_seed(2)
    X = torch.randint(-8, 9, (m, n), device="cuda", generator=gen).float().mul(2.0 ** -3).to(TYPES[kind])
    W = (torch.randn((p, n), device="cuda", generator=gen) * 0.08).to(TYPES[kind])
    y = torch.randint(0, p, (m,), device="cuda", generator=gen)
    _, lse = lm.cross_entropy(X, W, y)
    dX, _ = lm.cross_entropy_backward(torch.ones(m, device="cuda"), X, W, y, lse, dx_type=torch.float32)
    for _ in range(5):
        E = torch.randint(0, 2, (m, n), device="cuda", generator=gen).float() * 2 - 1
        up, down = ((X.float() + s * h * E).to(TYPES[kind]) for s in (1, -1))
        assert torch.equal(up.float() - down.float(), 2 * h * E)
        difference = (lm.cross_entropy(up, W, y)[0].double() - lm.cross_entropy(down, W, y)[0].double()) / (2 * h)
        along = (dX.double() * E).sum(1)
        # (dX: the slopes' rounding, half a step each of sum |d W|, about 2 sum |W_y|)
        limit = 0.01 * (1 + along.abs()) + 2 * HALF[kind] * W.double().abs().sum(1).max() * 2
        assert ((difference - along).abs() <= limit).all()


@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_ignored_rows_of_anything_and_targets_that_no_word_has(lm, kind):
    for m, n, p in ((9, 64, 100), (70, 1001, 3001), (300, 136, 2000)):
        X, W, y = layer(m, n, p, kind, 4, ignored=0.0)
        g = torch.rand(m, device="cuda") + 0.5
        ignored = torch.zeros(m, dtype=torch.bool, device="cuda")
        ignored[[1, 3, m - 1]] = True
        y[ignored] = IGNORE
        _, lse0 = lm.cross_entropy(X, W, y)
        want = lm.cross_entropy_backward(g, X, W, y, lse0)
        dirty, dirty_g = X.clone(), g.clone()
        dirty[1], dirty[3, 0], dirty[m - 1, n - 1] = float("nan"), float("inf"), float("nan")
        dirty_g[1], dirty_g[3], dirty_g[m - 1] = float("nan"), 1e30, float("inf")
        loss, lse = lm.cross_entropy(dirty, W, y)
        assert (loss[ignored] == 0).all() and torch.equal(lse[~ignored], lse0[~ignored])
        got = lm.cross_entropy_backward(dirty_g, dirty, W, y, lse)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and (got[0][ignored] == 0).all()
        # all rows ignored: nothing, and no NaN of a division by nothing
        none = torch.full_like(y, IGNORE)
        loss, lse = lm.cross_entropy(X, W, none)
        dX, dW = lm.cross_entropy_backward(g, X, W, none, lse)
        assert (loss == 0).all() and (dX == 0).all() and (dW == 0).all()
        # `ignore` may be a word
        first = y.clone()
        first[5] = 0
        loss, lse = lm.cross_entropy(X, W, first, ignore=0)
        want_loss, want_lse, _ = exact(X, W, torch.where(first == IGNORE, 1, first), ignore=0)
        assert loss[5] == 0 and torch.allclose(lse.double(), want_lse, atol=1e-4)
        for bad in (p, -1, 2 ** 40, -2 ** 62):
            wrong = y.clone()
            wrong[0] = bad
            loss, lse = lm.cross_entropy(X, W, wrong)
            assert torch.isnan(loss[0]) and torch.isfinite(loss[1:]).all() and torch.isfinite(lse).all()
            dX, dW = lm.cross_entropy_backward(g, X, W, wrong, lse)
            assert torch.isnan(dX[0]).all() and torch.equal(dX[1:], want[0][1:]) and torch.isnan(dW).all()


def test_strides_of_targets_and_of_g(lm):
    X, W, y = layer(100, 200, 500, "bf16", 6)
    wide = torch.full((100, 3), 10 ** 6, device="cuda")
    wide[:, 1] = y
    g = torch.full((1,), 0.25, device="cuda")
    loss, lse = lm.cross_entropy(X, W, wide[:, 1])
    assert torch.equal(loss, lm.cross_entropy(X, W, y)[0])
    a = lm.cross_entropy_backward(g.expand(100), X, W, wide[:, 1], lse)
    b = lm.cross_entropy_backward(g.repeat(100), X, W, y, lse)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    one = y[:1].expand(100)
    assert torch.equal(lm.cross_entropy(X, W, one)[0], lm.cross_entropy(X, W, one.contiguous())[0])


def test_gradients_into_others_and_added_to_what_is_there(lm):
    for m, n, p, kind in ((40, 100, 300, "bf16"), (300, 264, 1000, "f16"), (600, 1001, 1500, "bf16")):
        X, W, y = layer(m, n, p, kind, 7)
        g = torch.rand(m, device="cuda")
        _, lse = lm.cross_entropy(X, W, y)
        dX, dW = lm.cross_entropy_backward(g, X, W, y, lse, dw_type=torch.float32)
        for t in (torch.float32, TYPES[kind]):
            big_x = torch.full((m + 1, n + 3), 5.0, dtype=TYPES[kind], device="cuda")
            big_w = torch.randn((p + 1, n + 5), device="cuda").to(t)
            before = big_w.clone()
            lm.cross_entropy_backward(g, X, W, y, lse, dX=big_x[:m, 1:n + 1], dW=big_w[:p, 2:n + 2], beta=0.5)
            assert torch.equal(big_x[:m, 1:n + 1], dX) and (big_x[:, 0] == 5).all() and (big_x[:, n + 1:] == 5).all() and (big_x[m] == 5).all()
            want = dW.double() + 0.5 * before[:p, 2:n + 2].double()
            limit = HALF["f32" if t is torch.float32 else kind] * 1.01 * want.abs() + 2.0 ** -22 * (dW.double().abs() + before[:p, 2:n + 2].double().abs()) + 2.0 ** -24
            assert ((big_w[:p, 2:n + 2].double() - want).abs() <= limit).all()
            changed = big_w.clone()
            changed[:p, 2:n + 2] = before[:p, 2:n + 2]
            assert torch.equal(changed, before)
            nan = torch.full((p, n), float("nan"), dtype=t, device="cuda")
            lm.cross_entropy_backward(g, X, W, y, lse, dW=nan, need_dx=False)
            assert torch.isfinite(nan).all()


def test_no_tokens(lm):
    X, W, y = layer(3, 64, 100, "bf16", 8)
    X, y, g = X[:0], y[:0], torch.empty(0, device="cuda")
    loss, lse = lm.cross_entropy(X, W, y)
    assert loss.shape == lse.shape == (0,)
    dX, dW = lm.cross_entropy_backward(g, X, W, y, lse)
    assert dX.shape == (0, 64) and (dW == 0).all()
    kept = torch.ones((100, 64), device="cuda")
    lm.cross_entropy_backward(g, X, W, y, lse, dW=kept, beta=1.0)
    assert (kept == 1).all()
    lm.cross_entropy_backward(g, X, W, y, lse, dW=kept, beta=0.5)
    assert (kept == 0.5).all()


def test_a_vocabulary_in_several_pieces_and_tokens_in_several_rounds(lm):
    """300 tokens: slopes of 131072 words at a time.  2^22 - 256 words: parts of 512 tokens at a time."""
    for m, n, p, kind in ((300, 40, 300001, "f16"), (300, 64, 270000, "bf16")):
        X, W, y = layer(m, n, p, kind, 9, known=2.0)
        y[:3] = torch.tensor([p - 1, 131072, 131071], device="cuda")
        g = torch.ones(m, device="cuda") / m
        loss, lse = lm.cross_entropy(X, W, y)
        want, want_lse, size, d = exact(X, W, y, g)
        assert ((loss.double() - want).abs() <= 2 * size + 40 * 2.0 ** -24 * (1 + want_lse)).all()
        dX, dW = lm.cross_entropy_backward(g, X, W, y, lse)
        check_gradient(dX, d, W.double(), g.double(), size, kind, kind, False, "dX")
        check_gradient(dW, d, X.double(), g.double(), size, kind, kind, True, "dW")
        del d
    p = 2 ** 22 - 256
    X, W, y = layer(700, 8, p, "bf16", 10)
    y[650] = p - 1
    loss, lse = lm.cross_entropy(X, W, y)
    for part in (slice(0, 40), slice(500, 530), slice(640, 700)):
        want, want_lse, size = exact(X[part], W, y[part])
        assert ((loss[part].double() - want).abs() <= 2 * size + 40 * 2.0 ** -24 * (1 + want_lse)).all()


def test_a_workspace_of_the_users_and_one_too_small(lm):
    from paper_2409_13313_amd.ozimmu import OzimmuError
    for m, n, p, pad in ((5, 100, 3000, 0), (200, 1001, 2000, 1), (400, 2048, 3000, 0)):
        X, W, y = layer(m, n, p, "bf16", 11, pad)
        g = torch.rand(m, device="cuda")
        loss, lse = lm.cross_entropy(X, W, y)
        grads = lm.cross_entropy_backward(g, X, W, y, lse)
        for backward in (False, True):
            need = lm.cross_entropy_workspace_bytes(m, n, p, backward)
            room = torch.full((need + 256,), 255, dtype=torch.uint8, device="cuda")     # (NaN wherever it is read before it is written)
            if backward:
                got = lm.cross_entropy_backward(g, X, W, y, lse, workspace=room[:need])
                assert torch.equal(got[0], grads[0]) and torch.equal(got[1], grads[1])
                call = lambda: lm.cross_entropy_backward(g, X, W, y, lse, workspace=room[:need - 256])  # noqa: E731
            else:
                got = lm.cross_entropy(X, W, y, workspace=room[:need])
                assert torch.equal(got[0], loss) and torch.equal(got[1], lse)
                call = lambda: lm.cross_entropy(X, W, y, workspace=room[:need - 256])  # noqa: E731
            assert (room[need:] == 255).all()
            with pytest.raises(OzimmuError):
                call()


@pytest.mark.parametrize("m,n,p", [(1, 8, 16), (1, 96, 300), (3, 1001, 70), (20, 130, 500), (33, 64, 200), (48, 515, 1000)])
@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_rows_that_begin_at_odd_elements_beside_nan(lm, m, n, p, kind):
    """The same numbers wherever their rows begin, in memory that is full of NaN elsewhere."""
    X, W, y = layer(m, n, p, kind, m + n + p)

    def placed(t, begin, ld):
        room = torch.full((begin + len(t) * ld,), float("nan"), device="cuda", dtype=t.dtype)
        at = room.as_strided((len(t), n), (ld, 1), begin)
        at.copy_(t)
        return at
    even = n + n % 2 + 2                                        # (neither of whole 16 bytes where it matters which plan is taken, nor odd)
    even += 2 * (even % 8 == 0)
    want = lm.cross_entropy(placed(X, 2, even), placed(W, 2, even), y)
    loss, lse, size = exact(X, W, y)
    assert ((want[0].double() - loss).abs() <= 2 * size + 40 * 2.0 ** -24 * (1 + lse.abs())).all()
    for x, w in (((1, even), (1, even)), ((1, even + 1), (2, even)), ((2, even), (2, even + 1)), ((1, n + 1 - n % 2), (1, n + 1 - n % 2))):
        got = lm.cross_entropy(placed(X, *x), placed(W, *w), y)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), (x, w)
