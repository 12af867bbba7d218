"""The loss and its gradient where the vocabulary is taken in pieces for reasons of their own: many tokens, and rows that are laid out anew.

Bounds are those of test_gpu_lm_loss.py; sums over the tokens, of which there are more here, are off by (6 m / 32 + 8) roundings of 2^-23 of their terms."""
import pytest

torch = pytest.importorskip("torch")
from test_gpu_lm_loss import HALF, check_gradient, exact, layer, lm  # noqa: E402,F401

pytestmark = pytest.mark.gpu


# words at a time: 256 (from 262144 tokens on), 4352, 131072 (256 MB of rows laid out)
@pytest.mark.parametrize("m,n,p,pad,last", [(300000, 8, 600, 0, 256), (15000, 72, 6000, 0, 4352), (15000, 33, 5000, 1, 4352), (5, 1001, 140000, 1, 131072)])
@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_pieces(lm, m, n, p, pad, last, kind):  # noqa: F811
    X, W, y = layer(m, n, p, kind, m + n, pad)
    y[:3] = torch.tensor([p - 1, last - 1, last], device="cuda")
    g = torch.rand(m, device="cuda") + 0.5
    loss, lse = lm.cross_entropy(X, W, y)
    want, want_lse, size, d = exact(X, W, y, g)
    limit = 2 * size + 40 * 2.0 ** -24 * (1 + want_lse.abs())
    assert ((lse.double() - want_lse).abs() <= limit).all() and ((loss.double() - want).abs() <= limit).all()
    dX, dW = lm.cross_entropy_backward(g, X, W, y, lse, dw_type=torch.float32)
    check_gradient(dX, d, W.double(), g.double(), size, kind, kind, False, "dX")
    x, gd = X.double(), d * g.double().unsqueeze(1)
    p_of = (d + (d < 0)).abs()
    off_d = (HALF[kind] * d.abs() + 2.0 ** -40 + (size.unsqueeze(1) * 2 + 2.0 ** -20) * p_of) * g.double().unsqueeze(1)
    sums = gd.abs().t() @ x.abs()
    # (in FP16 what is held of a row of X is off by 2^-11 of itself, or 2^-21 of its largest)
    least = 2.0 ** -21 * gd.abs().t() @ x.abs().amax(1, keepdim=True)
    bound = off_d.t() @ x.abs() + (HALF[kind] + (6 * m / 32 + 8) * 2.0 ** -23) * sums + least
    off = (dW.double() - gd.t() @ x).abs()
    limit = bound + 2.0 ** -23 * (sums + bound)
    assert (off <= limit).all(), f"{(off / limit).max().item():.3g} of the bound"
    again = lm.cross_entropy_backward(g, X, W, y, lse, dw_type=torch.float32)
    assert torch.equal(again[0], dX) and torch.equal(again[1], dW)
