"""The example runs, its function hands torch's autograd the gradients of the formula, and what it stores is what it serves."""
import os
import runpy

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "lm_output_layer.py")


def test_example(monkeypatch, capsys):
    monkeypatch.setattr("sys.argv", ["lm_output_layer.py", "--steps", "5", "--tokens", "300", "--width", "200", "--words", "1000"])
    losses, scored, off = runpy.run_path(PATH)["main"]()
    assert all(l == l for l in losses) and scored == scored
    # (two roundings of a logit to BF16, of half a step each, and FP32 sums in another order)
    assert off <= 2.1 * 2.0 ** -8
    assert "bits a weight" in capsys.readouterr().out


def test_gradients_of_its_function():
    """Against torch's own in 64 bits.  Bounds: slopes and results in BF16, half a step (2^-8) each; sums of a few hundred terms of either sign, whose norm
    counts each rounding once."""
    Loss = runpy.run_path(PATH)["Loss"]
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((100, 64), device="cuda", generator=gen).bfloat16().requires_grad_()
    w = (torch.randn((500, 64), device="cuda", generator=gen) * 0.2).bfloat16().requires_grad_()
    y = torch.randint(0, 500, (100,), device="cuda", generator=gen)
    y[::7] = -100
    (3 * Loss.apply(x, w, y)).backward()
    xd, wd = (t.detach().double().cpu().requires_grad_() for t in (x, w))
    (3 * torch.nn.functional.cross_entropy(xd @ wd.t(), y.cpu())).backward()
    for got, want in ((x.grad, xd.grad), (w.grad, wd.grad)):
        assert (got.double().cpu() - want).norm() <= 2 * 2.0 ** -8 * want.norm()
