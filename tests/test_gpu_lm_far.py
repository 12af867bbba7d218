"""The loss and its gradient where numbers of one call are orders of magnitude apart, against the definition in 64 bits.

Bounds are those of test_gpu_lm_loss.py, of the words that carry a row's sum: words whose logits lie so far below that their exponentials are zero in 64 bits
too have no part in it, whatever their logits' own error is."""
import pytest

torch = pytest.importorskip("torch")
from test_gpu_lm_loss import HALF, IGNORE, TYPES, check_gradient, lm  # noqa: E402,F401

pytestmark = pytest.mark.gpu
# straight from memory, the same with rows at odd elements, and by tiles
SIZES = [(5, 64, 300, 0), (5, 200, 1000, 1), (300, 512, 8200, 0)]


def masked(m, n, p, kind, pad, seed, bias):
    """Column 0 of X is one, and every fifth word has `bias` there: it may not be taken.  Of the rows one in three has such a word as its target."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    X = torch.randn((m, n + pad), device="cuda", generator=gen).to(TYPES[kind])[:, :n]
    W = (torch.randn((p, n + pad), device="cuda", generator=gen) * n ** -0.5).to(TYPES[kind])[:, :n]
    X[:, 0] = 1
    W[::5, 0] = bias
    y = torch.randint(0, p // 5 - 1, (m,), device="cuda", generator=gen) * 5 + 1
    y[::3] -= 1
    y[4] = IGNORE
    return X, W, y


@pytest.mark.parametrize("m,n,p,pad", SIZES)
@pytest.mark.parametrize("kind,bias", [("bf16", -65504.0), ("bf16", -1e6), ("bf16", -1e9), ("bf16", float("-inf")), ("f16", -65504.0), ("f16", float("-inf"))])
def test_targets_far_below_the_other_words(lm, m, n, p, pad, kind, bias):  # noqa: F811
    X, W, y = masked(m, n, p, kind, pad, m + n, bias)
    x, w = X.double(), W.double()
    z = x @ w.t()
    lse = torch.logsumexp(z, 1)
    learnt = y != IGNORE
    at = torch.where(learnt, y, 1).unsqueeze(1)
    want = torch.where(learnt, lse - z.gather(1, at).squeeze(1), 0.0)
    part = (x.abs() @ w.abs().t()) * (6 * n / 32 + 8) * 2.0 ** -23
    part[:, ::5], of_target = 0, part.gather(1, at).squeeze(1)
    size = part.amax(1)
    loss, got = lm.cross_entropy(X, W, y)
    assert ((got.double() - lse).abs() <= size + 40 * 2.0 ** -24 * (1 + lse.abs())).all()
    finite = torch.isfinite(want)
    assert (loss[~finite] == float("inf")).all()
    limit = size + of_target + 40 * 2.0 ** -24 * (1 + lse.abs() + want.abs())
    assert ((loss.double() - want).abs() <= limit)[finite].all()
    d = (z - lse.unsqueeze(1)).exp()
    d.scatter_add_(1, at, torch.full_like(lse, -1.0).unsqueeze(1))
    d = torch.where(learnt.unsqueeze(1), d, 0.0)
    g = torch.rand(m, device="cuda") + 0.5
    dX, dW = lm.cross_entropy_backward(g, X, W, y, got, dw_type=torch.float32, dx_type=torch.float32)
    check_gradient(dW, d, x, g.double(), size, kind, "f32", True, "dW")
    w[::5, 0] = w[::5, 0].clamp(min=-1e30)
    first = 1 if bias == float("-inf") else 0                         # (no slope times an infinity is a number)
    check_gradient(dX[:, first:], d, w[:, first:], g.double(), size, kind, "f32", False, "dX")


@pytest.mark.parametrize("m,n,p,pad", SIZES)
@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_a_logit_that_is_infinite(lm, m, n, p, pad, kind):  # noqa: F811
    """Its row has neither a logarithm of a sum nor a loss that are numbers (infinity less infinity), whether it is the target's logit or not."""
    X, W, y = masked(m, n, p, kind, pad, m + n, -100.0)
    X[2, :] = 0
    X[2, 0] = 1                                                       # (a row in which no other element meets the infinity)
    for word in (int(y[2]), int(y[2]) + 1):
        V = W.clone()
        V[word, 0] = float("inf")
        loss, lse = lm.cross_entropy(X, V, y)
        learnt = y != IGNORE
        assert torch.isnan(loss[learnt]).all() and torch.isnan(lse).all() and (loss[~learnt] == 0).all(), word
