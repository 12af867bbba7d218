"""Tensors on another device than the current one, whose stream a call goes to, are refused by the binding of the microscaled 4-bit operators
(tensors and library are stand-ins: no GPU)."""
import pytest

torch = pytest.importorskip("torch")
from test_mx_refusals import LIB, Tensor as Bare  # noqa: E402
import os  # noqa: E402

pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libozimmu.so not built (run __graft_entry__.build())")


class Tensor(Bare):
    def __init__(self, *shape, at=0, **kw):
        super().__init__(*shape, **kw)
        self.device = torch.device("cuda", at)

    def new_empty(self, shape, dtype=None):
        return Tensor(*(shape if isinstance(shape, tuple) else (shape,)), dtype=dtype or self.dtype, at=self.device.index)


@pytest.fixture
def mx(monkeypatch):
    from paper_2409_13313_amd import mx, ozimmu

    class Library:
        def __init__(self):
            self.calls = []

        def __getattr__(self, name):
            return lambda *args: (self.calls.append(name), 0)[1]

    monkeypatch.setattr(mx, "_lib", Library())
    monkeypatch.setattr(ozimmu, "_stream", lambda: 0)
    monkeypatch.setattr(ozimmu, "_current_device", lambda: 1)
    monkeypatch.setattr(mx, "_several_devices", True)
    # (results that come without a tensor's new_empty)
    monkeypatch.setattr(torch, "empty", lambda shape, dtype=None, device=None: Tensor(*shape, dtype=dtype, at=device.index))
    return mx


def uint8(*shape, at):
    return Tensor(*shape, dtype=torch.uint8, at=at)


# a call, with its tensors made by f(number in the call, ...) so that one of them at a time can be elsewhere
CALLS = {
    "quantize": (1, lambda mx, f, P: mx.quantize(f(0, 20, 64), cols=True)),
    "dequantize": (1, lambda mx, f, P: mx.dequantize(P(0, 32, 64))),
    "dequantize into": (2, lambda mx, f, P: mx.dequantize(P(0, 32, 64), out=f(1, 32, 64))),
    "pack": (2, lambda mx, f, P: mx.pack(f(0, 4, 32, dtype=torch.uint8), f(1, 4, 2, dtype=torch.uint8))),
    "unpack": (1, lambda mx, f, P: mx.unpack(P(0, 32, 64))),
    "gemm": (2, lambda mx, f, P: mx.gemm(P(0, 20, 64), P(1, 32, 64))),
    "gemm into": (3, lambda mx, f, P: mx.gemm(P(0, 20, 64), P(1, 32, 64), beta=1.0, D=f(2, 20, 32))),
    "linear": (2, lambda mx, f, P: mx.linear(f(0, 20, 64), P(1, 32, 64))),
    "linear into": (4, lambda mx, f, P: mx.linear(f(0, 20, 64), P(1, 32, 64), D=f(2, 20, 32), workspace=f(3, 4096, dtype=torch.uint8))),
    "gradient": (3, lambda mx, f, P: mx.linear_backward(f(0, 20, 32), f(1, 20, 64), P(2, 64, 32))),
    "gradient into": (6, lambda mx, f, P: mx.linear_backward(f(0, 20, 32), f(1, 20, 64), P(2, 64, 32), dX=f(3, 20, 64), dW=f(4, 32, 64),
                                                             workspace=f(5, 4096, dtype=torch.uint8))),
}


@pytest.mark.parametrize("call", list(CALLS))
def test_one_device_and_the_current_one(mx, call):
    count, run = CALLS[call]

    def go(where):
        mx._lib.calls.clear()
        run(mx, lambda i, *shape, **kw: Tensor(*shape, at=where[i], **kw),
            lambda i, rows, n: mx._empty(rows, n, Tensor(1, 1, at=where[i])))
        return [c for c in mx._lib.calls if not c.endswith("bytes")]

    assert len(go([1] * count)) == 1
    for elsewhere in [[0] * count] + [[1] * i + [0] + [1] * (count - i - 1) for i in range(count)]:
        with pytest.raises(ValueError, match="current device"):
            go(elsewhere)
        assert all(c.endswith("bytes") for c in mx._lib.calls), elsewhere


def test_one_device_alone_needs_no_look(mx, monkeypatch):
    monkeypatch.setattr(mx, "_several_devices", False)
    mx.quantize(Tensor(20, 64))
    assert "ozimmu_mx_quantize" in mx._lib.calls
