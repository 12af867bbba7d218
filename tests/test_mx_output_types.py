"""An output that is handed over and a type that is asked for have to agree (tensors and library are stand-ins: no GPU)."""
import os

import pytest

torch = pytest.importorskip("torch")
from test_mx_refusals import LIB, Tensor, launched, mx  # noqa: E402,F401

pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libozimmu.so not built (run __graft_entry__.build())")

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
CALLS = {"linear": lambda mx, P, D, **kw: mx.linear(Tensor(20, 64), P(32, 64), D=D, **kw),
         "gemm": lambda mx, P, D, **kw: mx.gemm(P(20, 64), P(32, 64), D=D, **kw),
         "dequantize": lambda mx, P, D, **kw: mx.dequantize(P(20, 32), out=D, **kw)}
TYPE_AT = {"linear": 9, "gemm": 8, "dequantize": 0}


@pytest.mark.parametrize("call", list(CALLS))
def test_type_and_output(mx, call):  # noqa: F811
    packed = lambda rows, n: mx._empty(rows, n, Tensor(1, 1))  # noqa: E731

    def kind(D, **kw):
        mx._lib.calls.clear()
        out = CALLS[call](mx, packed, D, **kw)
        (_, args), = launched(mx)
        return out.dtype, args[TYPE_AT[call]]

    for number, t in ((0, F32), (1, BF16), (2, F16)):
        assert kind(None, dtype=t) == (t, number)
        assert kind(Tensor(20, 32, dtype=t)) == (t, number)
        assert kind(Tensor(20, 32, dtype=t), dtype=t) == (t, number)
        mx._lib.calls.clear()
        for other in {F32, BF16, F16} - {t}:
            with pytest.raises(ValueError, match="output of"):
                CALLS[call](mx, packed, Tensor(20, 32, dtype=t), dtype=other)
        assert launched(mx) == []
    assert kind(None) == (F32, 0)          # linear: the type of X


def test_type_of_x(mx):  # noqa: F811
    W = mx._empty(32, 64, Tensor(1, 1))
    assert mx.linear(Tensor(20, 64, dtype=BF16), W).dtype is BF16
    # gradients that are handed over: in whatever type each of them is
    dX, dW = mx.linear_backward(Tensor(20, 32, dtype=BF16), Tensor(20, 64, dtype=BF16), mx._empty(64, 32, Tensor(1, 1)),
                                dX=Tensor(20, 64, dtype=F16), dW=Tensor(32, 64, dtype=BF16))
    assert dX.dtype is F16 and dW.dtype is BF16
