"""The microscaled layer and its gradient do not record operations for torch's autograd: a tensor whose gradient would be lost silently is refused
(tensors and library are stand-ins: no GPU)."""
import os

import pytest

torch = pytest.importorskip("torch")
from test_mx_refusals import LIB, Tensor as Bare, launched, mx  # noqa: E402,F401

pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libozimmu.so not built (run __graft_entry__.build())")


class Tensor(Bare):
    def __init__(self, *shape, requires_grad=False, **kw):
        super().__init__(*shape, **kw)
        self.requires_grad = requires_grad


def calls(mx, **grad):
    t = lambda name, *shape: Tensor(*shape, requires_grad=grad.get(name, False))  # noqa: E731
    packed = lambda rows, n: mx._empty(rows, n, Bare(1, 1))  # noqa: E731
    return {"linear": lambda: mx.linear(t("X", 20, 64), packed(32, 64)),
            "both gradients": lambda: mx.linear_backward(t("G", 20, 32), t("X", 20, 64), packed(64, 32)),
            "dX": lambda: mx.linear_backward(t("G", 20, 32), None, packed(64, 32)),
            "dW": lambda: mx.linear_backward(t("G", 20, 32), t("X", 20, 64), None)}


@pytest.mark.parametrize("call,tensor", [("linear", "X"), ("both gradients", "X"), ("both gradients", "G"), ("dX", "G"), ("dW", "X"), ("dW", "G")])
def test_a_gradient_that_would_be_lost(mx, call, tensor):  # noqa: F811
    with pytest.raises(ValueError, match="requires a gradient"):
        calls(mx, **{tensor: True})[call]()
    assert launched(mx) == []
    # as in the forward and the backward pass of a function of the user's own, where torch records nothing
    with torch.no_grad():
        calls(mx, **{tensor: True})[call]()
    assert len(launched(mx)) == 1
    calls(mx)[call]()
    assert len(launched(mx)) == 2


def test_quantisation_takes_weights_that_are_trained(mx):  # noqa: F811
    """(its result is no tensor: nothing that could pass for having a gradient)"""
    mx.quantize(Tensor(32, 64, requires_grad=True), cols=True)
    assert len(launched(mx)) == 1
