"""What the microscaled 4-bit operators refuse, in the C ABI (no GPU: every call fails its checks, or has nothing to do) and in the binding
(tensors and library are stand-ins)."""
import ctypes
import os

import pytest

torch = pytest.importorskip("torch")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2409_13313_amd", "libozimmu.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libozimmu.so not built (run __graft_entry__.build())")

NULL, DIM, ROOM, TYPE, WAY = -1, -2, -4, -6, -7
AT = 4096            # an address that is never looked at
F32, BF16 = 0, 1


@pytest.fixture(scope="module")
def lib():
    from paper_2409_13313_amd import mx
    return mx._lib


def test_header_and_binding_agree():
    import re
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "ozimmu_mx.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(ozimmu_mx_[a-z_]+)\s*\(", text)))
    from paper_2409_13313_amd import mx
    assert names == sorted(mx.EXPORTS)
    for name in names:
        args = re.search(name + r"\s*\((.*?)\);", text, flags=re.S).group(1)
        assert len(args.split(",")) == len(getattr(mx._lib, name).argtypes), name


def test_quantize(lib):
    q = lib.ozimmu_mx_quantize
    assert q(7, 4, 4, AT, 4, AT, None, None) == TYPE and q(-1, 4, 4, AT, 4, AT, None, None) == TYPE
    assert q(F32, 4, 4, AT + 2, 4, AT, None, None) == TYPE and q(BF16, 4, 4, AT + 1, 4, AT, None, None) == TYPE
    assert q(F32, -1, 4, AT, 4, AT, None, None) == DIM and q(F32, 4, -4, AT, 4, AT, None, None) == DIM
    assert q(F32, 4, 4, AT, 3, AT, None, None) == DIM and q(F32, 4, 4, AT, 2 ** 40, AT, None, None) == DIM
    assert q(F32, 2 ** 22, 4, AT, 4, AT, None, None) == DIM            # rows of the packed form
    assert q(F32, 4, 2 ** 22, AT, 2 ** 22, None, AT, None) == DIM
    assert q(F32, 4, 2 ** 29 + 1, AT, 2 ** 30, AT, None, None) == DIM  # its inner dimension
    assert q(F32, 4, 4, None, 4, AT, None, None) == NULL and q(F32, 4, 4, AT, 4, None, None, None) == NULL
    assert q(F32, 4, 4, AT, 4, AT + 16, None, None) == ROOM and q(F32, 4, 4, AT, 4, AT, AT + 128, None) == ROOM
    assert q(F32, 0, 4, None, 4, None, None, None) == 0 and q(F32, 4, 0, None, 0, None, None, None) == 0


def test_dequantize_and_plain_layout(lib):
    d = lib.ozimmu_mx_dequantize
    assert d(3, 4, 4, AT, AT, 4, None) == TYPE and d(F32, 4, 4, AT, AT, 3, None) == DIM
    assert d(F32, 4, 4, None, AT, 4, None) == NULL and d(F32, 4, 4, AT, None, 4, None) == NULL and d(F32, 4, 4, AT + 64, AT, 4, None) == ROOM
    assert d(F32, 0, 4, None, None, 4, None) == 0
    for f in (lambda c, ldc, s, lds, p: lib.ozimmu_mx_pack(4, 40, c, ldc, s, lds, p, None),
              lambda c, ldc, s, lds, p: lib.ozimmu_mx_unpack(4, 40, p, c, ldc, s, lds, None)):
        assert f(AT, 31, AT, 2, AT) == DIM and f(AT, 32, AT, 1, AT) == DIM
        assert f(None, 32, AT, 2, AT) == NULL and f(AT, 32, None, 2, AT) == NULL and f(AT, 32, AT, 2, None) == NULL
        assert f(AT, 32, AT, 2, AT + 8) == ROOM


def test_products(lib):
    g = lambda m=4, n=4, p=4, A=AT, B=AT, t=F32, D=AT, ldd=4, way=-1: lib.ozimmu_mx_gemm_way(way, m, n, p, 1.0, A, B, 0.0, t, D, ldd, None)  # noqa: E731
    assert g(m=-1) == DIM and g(n=-1) == DIM and g(p=2 ** 22, ldd=2 ** 22) == DIM and g(ldd=3) == DIM
    assert g(A=None) == NULL and g(B=None) == NULL and g(D=None) == NULL
    assert g(A=AT + 4) == ROOM and g(B=AT + 4) == ROOM and g(t=5) == TYPE and g(D=AT + 1) == TYPE
    assert g(way=1) == WAY and g(way=2, n=640) == WAY and g(way=9, n=4096) == WAY and g(way=1, n=4096, ldd=2 ** 24) == WAY
    assert g(m=0) == 0 and g(p=0, ldd=0) == 0
    assert lib.ozimmu_mx_gemm(4, 4, 4, 1.0, AT, None, 0.0, F32, AT, 4, None) == NULL

    def lin(m=100, n=64, p=64, xt=BF16, X=AT, ldx=64, W=AT, t=BF16, D=AT, ldd=64, ws=AT, size=1 << 30):
        return lib.ozimmu_mx_linear(m, n, p, 1.0, xt, X, ldx, W, 0.0, t, D, ldd, ws, size, None)
    assert lin(xt=4) == TYPE and lin(t=4) == TYPE and lin(X=AT + 1) == TYPE and lin(ldx=63) == DIM and lin(ldd=63) == DIM
    assert lin(X=None) == NULL and lin(W=None) == NULL and lin(D=None) == NULL and lin(W=AT + 1) == ROOM
    # (100 rows through 64 x 64 in two launches: X is packed in the workspace)
    assert lin(ws=None) == NULL and lin(size=16) == ROOM and lin(ws=AT + 16) == ROOM
    assert lin(m=0) == 0


def test_gradient(lib):
    def back(m=20, n=64, p=32, t=BF16, G=AT, ldg=32, X=AT, ldx=64, Wt=AT, tx=BF16, dX=AT, lddx=64, tw=F32, dW=AT, lddw=64, ws=AT, size=1 << 30):
        return lib.ozimmu_mx_linear_backward(m, n, p, 1.0, t, G, ldg, X, ldx, Wt, 0.0, tx, dX, lddx, 0.0, tw, dW, lddw, ws, size, None)
    assert back(m=-1) == DIM and back(ldg=31) == DIM and back(ldx=63) == DIM and back(lddx=63) == DIM and back(lddw=63) == DIM
    assert back(t=3) == TYPE and back(tx=3) == TYPE and back(tw=3) == TYPE
    assert back(G=None) == NULL and back(X=None) == NULL and back(Wt=None) == NULL and back(ws=None) == NULL
    assert back(Wt=AT + 2) == ROOM and back(size=17) == ROOM and back(ws=AT + 1) == ROOM
    assert back(dX=None, dW=None) == 0                                      # nothing asked for
    assert back(m=0, G=None, X=None, Wt=AT, dX=None, dW=None, ws=None) == 0


class Tensor:
    """A tensor as far as the binding looks at one."""
    def __init__(self, *shape, ld=None, dtype=torch.float32, is_cuda=True, unit=1):
        self.shape, self.dtype, self.is_cuda = shape, dtype, is_cuda
        self.strides = (shape[-1] if ld is None else ld, unit) if len(shape) == 2 else (1,) * len(shape)

    def dim(self):
        return len(self.shape)

    def stride(self, i=None):
        return self.strides if i is None else self.strides[i]

    def data_ptr(self):
        return AT

    def numel(self):
        return 1 << 40

    def is_contiguous(self):
        return True

    def new_empty(self, shape, dtype=None):
        return Tensor(*(shape if isinstance(shape, tuple) else (shape,)), dtype=dtype or self.dtype)


@pytest.fixture
def mx(monkeypatch):
    from paper_2409_13313_amd import mx, ozimmu

    class Library:
        calls = []

        def __getattr__(self, name):
            return lambda *args: self.calls.append((name, args)) or 0

    library = Library()
    library.calls.clear()
    monkeypatch.setattr(mx, "_lib", library)
    monkeypatch.setattr(ozimmu, "_stream", lambda: 0)
    return mx


def launched(mx):
    return [c for c in mx._lib.calls if not c[0].endswith("bytes")]


def test_binding_refuses(mx):
    packed = lambda rows, n: mx._empty(rows, n, Tensor(1, 1))  # noqa: E731
    X, G, W, Wt = Tensor(20, 64), Tensor(20, 32), packed(32, 64), packed(64, 32)
    bad = [lambda: mx.quantize(Tensor(20, 64, dtype=torch.float64)), lambda: mx.quantize(Tensor(20, 64, is_cuda=False)),
           lambda: mx.quantize(Tensor(20, 64, unit=2)), lambda: mx.quantize(Tensor(20, 64, ld=63)), lambda: mx.quantize(Tensor(20)),
           lambda: mx.quantize(X, rows=False), lambda: mx.dequantize(X), lambda: mx.dequantize(W, torch.int32),
           lambda: mx.dequantize(W, out=Tensor(32, 63)),
           lambda: mx.linear(Tensor(20, 63), W), lambda: mx.linear(X, Tensor(32, 64)), lambda: mx.linear(X, W, D=Tensor(20, 33)),
           lambda: mx.linear(X, W, D=Tensor(20, 32, is_cuda=False)), lambda: mx.linear(X, W, beta=1.0), lambda: mx.linear(X, W, dtype=torch.float64),
           lambda: mx.linear(X, W, workspace=Tensor(4096)),
           lambda: mx.gemm(W, Wt), lambda: mx.gemm(W, W, D=Tensor(31, 32)), lambda: mx.gemm(X, W), lambda: mx.gemm(W, W, beta=0.5),
           lambda: mx.linear_backward(G, None, None), lambda: mx.linear_backward(G, Tensor(19, 64), Wt),
           lambda: mx.linear_backward(G, Tensor(20, 64, dtype=torch.bfloat16), Wt), lambda: mx.linear_backward(G, X, W),
           lambda: mx.linear_backward(G, X, None, dX=X), lambda: mx.linear_backward(G, None, Wt, dW=X),
           lambda: mx.linear_backward(G, X, Wt, dX=Tensor(20, 63)), lambda: mx.linear_backward(G, X, Wt, beta_w=1.0),
           lambda: mx.pack(Tensor(4, 32, dtype=torch.uint8), Tensor(4, 2, dtype=torch.uint8), 65),
           lambda: mx.pack(Tensor(4, 31, dtype=torch.uint8), Tensor(4, 2, dtype=torch.uint8)),
           lambda: mx.pack(Tensor(4, 32), Tensor(4, 2, dtype=torch.uint8)),
           lambda: mx.pack(Tensor(4, 32, dtype=torch.uint8, unit=2), Tensor(4, 2, dtype=torch.uint8)),
           lambda: mx.Packed(Tensor(10), 4, 4)]
    mx._lib.calls.clear()
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
        assert launched(mx) == [], i


def test_binding_hands_over_sizes_and_leading_dimensions(mx):
    W, Wt = mx._empty(32, 64, Tensor(1, 1)), mx._empty(64, 32, Tensor(1, 1))
    mx._lib.calls.clear()
    D = mx.linear(Tensor(20, 64, ld=70, dtype=torch.bfloat16), W)
    (name, args), = launched(mx)
    assert name == "ozimmu_mx_linear" and args[:3] == (20, 64, 32) and args[4] == 1 and args[6] == 70 and args[9] == 1 and args[11] == 32
    assert D.shape == (20, 32) and D.dtype is torch.bfloat16
    mx._lib.calls.clear()
    dX, dW = mx.linear_backward(Tensor(20, 32, ld=33), Tensor(20, 64, ld=65), Wt, dX=Tensor(20, 64, ld=66))
    (name, args), = launched(mx)
    assert args[:3] == (20, 64, 32) and args[6] == 33 and args[8] == 65 and args[13] == 66 and args[17] == 64 and args[15] == 0
    assert dW.shape == (32, 64) and dW.dtype is torch.float32


def test_status_strings():
    from paper_2409_13313_amd import ozimmu
    assert "type" in ozimmu.status_string(TYPE) and "way" in ozimmu.status_string(WAY)
