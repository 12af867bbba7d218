"""The example trains, stores, loads and serves a layer."""
import os
import runpy

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_example(monkeypatch, capsys):
    monkeypatch.setattr("sys.argv", ["mx_linear.py", "--steps", "20", "--tokens", "1024", "--inputs", "200", "--outputs", "96"])
    losses, rel = runpy.run_path(os.path.join(ROOT, "examples", "mx_linear.py"))["main"]()
    # the rounding of operands leaves an error of its own (about a tenth of each value); the rest is learnt
    assert losses[-1] < 0.1 * losses[0] and rel < 0.35
    assert "bits a weight" in capsys.readouterr().out
