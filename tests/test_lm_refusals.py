"""What the operators around the output layer refuse, in the C ABI (no GPU: every call fails its checks, or has nothing to do) and in the binding
(tensors and library are stand-ins); on which device and while torch records; what the binding hands over."""
import os
import re

import pytest

torch = pytest.importorskip("torch")
from test_mx_refusals import LIB, Tensor as Bare  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libozimmu.so not built (run __graft_entry__.build())")

NULL, DIM, ROOM, TYPE, WAY = -1, -2, -4, -6, -7
AT = 4096            # an address that is never looked at
F32, BF16, F16 = 0, 1, 2


@pytest.fixture(scope="module")
def lib():
    from paper_2409_13313_amd import lm
    return lm._lib


def test_header_and_binding_agree():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "ozimmu_lm.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(ozimmu_lm_[a-z_]+)\s*\(", text)))
    from paper_2409_13313_amd import lm
    assert names == sorted(lm.EXPORTS)
    for name in names:
        args = re.search(name + r"\s*\((.*?)\);", text, flags=re.S).group(1)
        assert len(args.split(",")) == len(getattr(lm._lib, name).argtypes), name


def test_weights(lib):
    q = lambda t=F32, p=4, n=40, W=AT, ld=40, group=32, zeros=1, st=F16, P=AT: lib.ozimmu_lm_quantize(t, p, n, W, ld, group, zeros, st, P, None)  # noqa: E731
    assert q(t=3) == TYPE and q(t=-1) == TYPE and q(st=F32) == TYPE and q(W=AT + 2) == TYPE and q(t=BF16, W=AT + 1) == TYPE
    assert q(p=-1) == DIM and q(n=-1) == DIM and q(ld=39) == DIM and q(p=2 ** 22) == DIM and q(n=2 ** 20 + 1, ld=2 ** 21) == DIM and q(group=48) == DIM
    assert q(ld=2 ** 40) == DIM and q(p=2 ** 22 - 256, ld=2 ** 39) == DIM
    assert q(W=None) == NULL and q(P=None) == NULL and q(P=AT + 16) == ROOM
    assert q(p=0, W=None, P=None) == 0 and q(n=0, W=None, P=None) == 0
    d = lambda t=F32, p=4, n=40, group=32, st=F16, P=AT, W=AT, ld=40: lib.ozimmu_lm_dequantize(t, p, n, group, 0, st, P, W, ld, None)  # noqa: E731
    assert d(t=5) == TYPE and d(st=0) == TYPE and d(group=0) == DIM and d(ld=39) == DIM and d(P=None) == NULL and d(W=None) == NULL and d(P=AT + 8) == ROOM
    for f in (lambda c=AT, ldc=20, s=AT, lds=2, z=AT, ldz=2, P=AT, n=40, group=32: lib.ozimmu_lm_pack(4, n, group, c, ldc, s, lds, z, ldz, P, None),
              lambda c=AT, ldc=20, s=AT, lds=2, z=AT, ldz=2, P=AT, n=40, group=32: lib.ozimmu_lm_unpack(4, n, group, P, c, ldc, s, lds, z, ldz, None)):
        assert f(ldc=19) == DIM and f(lds=1) == DIM and f(ldz=1) == DIM and f(group=256) == DIM and f(n=41) == DIM
        assert f(c=None) == NULL and f(s=None) == NULL and f(P=None) == NULL and f(P=AT + 1) == ROOM and f(s=AT + 1) == TYPE
        assert f(z=None, ldz=0, P=None) == NULL                     # (without zero points, ldz is not looked at)
    assert lib.ozimmu_lm_bytes(16, 128, 128, 0) > 1024 + 32 and lib.ozimmu_lm_bytes(16, 128, 100, 0) == 0 and lib.ozimmu_lm_bytes(-1, 4, 32, 0) == 0


def test_linear(lib):
    def lin(m=700, n=2048, p=2048, xt=BF16, X=AT, ldx=2048, group=64, st=F16, W=AT, t=BF16, D=AT, ldd=2048, ws=AT, size=1 << 40, way=-1):
        return lib.ozimmu_lm_linear_way(way, m, n, p, 1.0, xt, X, ldx, group, 0, st, W, 0.0, t, D, ldd, ws, size, None)
    assert lin(xt=F32) == TYPE and lin(xt=3) == TYPE and lin(t=3) == TYPE and lin(X=AT + 1) == TYPE and lin(st=F32) == TYPE
    assert lin(m=-1) == DIM and lin(n=0, ldx=0) == DIM and lin(ldx=2047) == DIM and lin(ldd=2047) == DIM and lin(group=7) == DIM and lin(m=2 ** 22) == DIM
    assert lin(X=None) == NULL and lin(W=None) == NULL and lin(D=None) == NULL and lin(W=AT + 4) == ROOM
    assert lin(way=3) == WAY and lin(way=-2) == WAY
    for way in (-1, 1):                                              # (700 rows take a workspace)
        assert lin(ws=None, way=way) == NULL and lin(size=16, way=way) == ROOM and lin(ws=AT + 16, way=way) == ROOM
    assert lin(m=0, X=None, D=None, ws=None) == 0 and lin(p=0, W=None, D=None, ws=None, ldd=0) == 0
    assert lib.ozimmu_lm_linear(4, 4, 4, 1.0, BF16, AT, 3, 32, 0, F16, AT, 0.0, BF16, AT, 4, None, 0, None) == DIM


def test_loss(lib):
    def loss(m=20, n=64, p=100, t=BF16, X=AT, ldx=64, W=AT, ldw=64, y=AT, sy=1, l=AT, e=AT, ws=AT, size=1 << 40):  # noqa: E741
        return lib.ozimmu_lm_cross_entropy(t, m, n, p, X, ldx, W, ldw, y, sy, -100, l, e, ws, size, None)
    assert loss(t=F32) == TYPE and loss(t=4) == TYPE and loss(X=AT + 1) == TYPE and loss(W=AT + 1) == TYPE and loss(y=AT + 4) == TYPE and loss(l=AT + 2) == TYPE
    assert loss(m=-1) == DIM and loss(n=0) == DIM and loss(p=0) == DIM and loss(p=2 ** 22) == DIM and loss(ldx=63) == DIM and loss(ldw=63) == DIM
    assert loss(sy=-1) == DIM and loss(m=2 ** 15, n=2 ** 16, ldx=2 ** 16, ldw=2 ** 16) == DIM    # (tokens x elements from 2^31 on)
    assert loss(X=None) == NULL and loss(W=None) == NULL and loss(y=None) == NULL and loss(l=None) == NULL and loss(e=None) == NULL and loss(ws=None) == NULL
    assert loss(size=17) == ROOM and loss(ws=AT + 8) == ROOM
    assert loss(m=0, X=None, y=None, l=None, e=None, ws=None) == 0
    assert lib.ozimmu_lm_cross_entropy_workspace_bytes(0, 64, 100) == 0 and lib.ozimmu_lm_cross_entropy_workspace_bytes(5, 0, 100) == 0


def test_gradient(lib):
    def back(m=20, n=64, p=100, t=BF16, g=AT, sg=1, X=AT, ldx=64, W=AT, ldw=64, y=AT, sy=1, e=AT, tx=BF16, dX=AT, lddx=64, tw=F32, dW=AT, lddw=64, ws=AT,
             size=1 << 40):
        return lib.ozimmu_lm_cross_entropy_backward(t, m, n, p, g, sg, X, ldx, W, ldw, y, sy, -100, e, tx, dX, lddx, 0.0, tw, dW, lddw, ws, size, None)
    assert back(t=F32) == TYPE and back(tx=3) == TYPE and back(tw=3) == TYPE and back(g=AT + 2) == TYPE and back(e=AT + 1) == TYPE and back(y=AT + 4) == TYPE
    assert back(dW=AT + 2) == TYPE and back(dX=AT + 1) == TYPE
    assert back(m=-1) == DIM and back(n=0) == DIM and back(p=0) == DIM and back(ldx=63) == DIM and back(ldw=63) == DIM and back(lddx=63) == DIM
    assert back(lddw=63) == DIM and back(sg=-1) == DIM and back(sy=-1) == DIM
    assert back(g=None) == NULL and back(X=None) == NULL and back(W=None) == NULL and back(y=None) == NULL and back(e=None) == NULL and back(ws=None) == NULL
    assert back(size=17) == ROOM and back(ws=AT + 128) == ROOM
    assert back(dX=None, dW=None) == 0 and back(m=0, g=None, X=None, y=None, e=None, dW=None, ws=None) == 0


class Tensor(Bare):
    def __init__(self, *shape, at=0, requires_grad=False, steps=None, **kw):
        super().__init__(*shape, **kw)
        self.device, self.requires_grad = torch.device("cuda", at), requires_grad
        if steps is not None:
            self.strides = steps

    def new_empty(self, shape, dtype=None):
        return Tensor(*(shape if isinstance(shape, tuple) else (shape,)), dtype=dtype or self.dtype, at=self.device.index)


B, I64, U8 = torch.bfloat16, torch.int64, torch.uint8


@pytest.fixture
def lm(monkeypatch):
    from paper_2409_13313_amd import lm, mx, ozimmu

    class Library:
        def __init__(self):
            self.calls = []

        def __getattr__(self, name):
            return lambda *args: (self.calls.append((name, args)), 4096 if name.endswith("bytes") else 0)[1]

    monkeypatch.setattr(lm, "_lib", Library())
    monkeypatch.setattr(ozimmu, "_stream", lambda: 0)
    monkeypatch.setattr(ozimmu, "_current_device", lambda: 1)
    monkeypatch.setattr(mx, "_several_devices", False)
    return lm


def launched(lm):
    return [c for c in lm._lib.calls if not c[0].endswith("bytes")]


def packed(lm, rows=32, n=64, at=0):
    return lm._empty(rows, n, 32, True, torch.float16, Tensor(1, 1, at=at))


def test_binding_refuses(lm):
    X, W, y, v = Tensor(20, 64, dtype=B), Tensor(100, 64, dtype=B), Tensor(20, dtype=I64), Tensor(20)
    P = packed(lm)
    bad = [lambda: lm.quantize(Tensor(4, 64, dtype=torch.float64)), lambda: lm.quantize(X, group=48), lambda: lm.quantize(X, scale_type=torch.float32),
           lambda: lm.quantize(Tensor(4, 64, is_cuda=False)), lambda: lm.quantize(Tensor(4, 64, unit=2)), lambda: lm.dequantize(X),
           lambda: lm.dequantize(P, torch.int32), lambda: lm.dequantize(P, out=Tensor(32, 63)), lambda: lm.unpack(X),
           lambda: lm.pack(Tensor(4, 32, dtype=U8), Tensor(4, 1)), lambda: lm.pack(Tensor(4, 32, dtype=U8), Tensor(4, 2, dtype=torch.float16)),
           lambda: lm.pack(Tensor(4, 32), Tensor(4, 1, dtype=torch.float16)), lambda: lm.pack(Tensor(4, dtype=U8), Tensor(4, 1, dtype=torch.float16)),
           lambda: lm.pack(Tensor(4, 32, dtype=U8), Tensor(4, 1, dtype=torch.float16), Tensor(4, 1)),
           lambda: lm.pack(Tensor(4, 32, dtype=U8), Tensor(4, 1, dtype=torch.float16), n=62), lambda: lm.pack(Tensor(4, 32, dtype=U8), Tensor(4, 1, dtype=B), group=16),
           lambda: lm.linear(Tensor(20, 64), P), lambda: lm.linear(Tensor(20, 63, dtype=B), P), lambda: lm.linear(X, W), lambda: lm.linear(X, P, beta=1.0),
           lambda: lm.linear(X, P, D=Tensor(20, 33)), lambda: lm.linear(X, P, dtype=torch.float64), lambda: lm.linear(X, P, workspace=Tensor(4096)),
           lambda: lm.linear(X, P, B, D=Tensor(20, 32)),
           lambda: lm.cross_entropy(Tensor(20, 64), W, y), lambda: lm.cross_entropy(X, Tensor(100, 64), y), lambda: lm.cross_entropy(X, Tensor(100, 63, dtype=B), y),
           lambda: lm.cross_entropy(X, Tensor(100, 64, dtype=torch.float16), y), lambda: lm.cross_entropy(X, W, Tensor(19, dtype=I64)),
           lambda: lm.cross_entropy(X, W, Tensor(20, dtype=torch.int32)), lambda: lm.cross_entropy(X, W, Tensor(20, 1, dtype=I64)),
           lambda: lm.cross_entropy(X, W, y, loss=Tensor(20, steps=(2,))), lambda: lm.cross_entropy(X, W, y, lse=Tensor(21)),
           lambda: lm.cross_entropy(X, W, y, workspace=Tensor(4096)),
           lambda: lm.cross_entropy_backward(Tensor(20, dtype=B), X, W, y, v), lambda: lm.cross_entropy_backward(v, X, W, y, Tensor(20, steps=(2,))),
           lambda: lm.cross_entropy_backward(v, X, W, y, Tensor(19)), lambda: lm.cross_entropy_backward(v, X, W, y, v, need_dx=False, need_dw=False),
           lambda: lm.cross_entropy_backward(v, X, W, y, v, need_dx=False, dX=X), lambda: lm.cross_entropy_backward(v, X, W, y, v, need_dw=False, dW=W),
           lambda: lm.cross_entropy_backward(v, X, W, y, v, beta=1.0), lambda: lm.cross_entropy_backward(v, X, W, y, v, dX=Tensor(20, 63)),
           lambda: lm.cross_entropy_backward(v, X, W, y, v, dw_type=torch.float64),
           lambda: lm.Packed(Tensor(10, dtype=U8), 4, 4, 33, True, B), lambda: lm.Packed(Tensor(10), 4, 4, 32, True, B)]
    lm._lib.calls.clear()
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
        assert launched(lm) == [], i


def test_binding_hands_over_sizes_strides_and_types(lm):
    P = packed(lm)
    lm._lib.calls.clear()
    D = lm.linear(Tensor(20, 64, ld=70, dtype=B), P)
    (name, args), = launched(lm)
    assert name == "ozimmu_lm_linear_way" and args[0] == -1 and args[1:4] == (20, 64, 32) and args[5] == 1 and args[7] == 70
    assert args[8:11] == (32, True, 2) and args[13] == 1 and args[15] == 32 and D.shape == (20, 32) and D.dtype is B
    lm._lib.calls.clear()
    y, g = Tensor(20, dtype=I64, steps=(3,)), Tensor(20, steps=(0,))
    X, W = Tensor(20, 64, ld=65, dtype=B), Tensor(100, 64, ld=66, dtype=B)
    loss, lse = lm.cross_entropy(X, W, y, ignore=7)
    (name, args), = launched(lm)
    assert args[:4] == (1, 20, 64, 100) and args[5] == 65 and args[7] == 66 and args[9] == 3 and args[10] == 7 and loss.dtype is lse.dtype is torch.float32
    lm._lib.calls.clear()
    dX, dW = lm.cross_entropy_backward(g, X, W, y, lse, dW=Tensor(100, 64, ld=68), beta=1.0)
    (name, args), = launched(lm)
    assert args[:4] == (1, 20, 64, 100) and args[5] == 0 and args[7] == 65 and args[9] == 66 and args[11] == 3 and args[14] == 1 and args[16] == 64
    assert args[17] == 1.0 and args[18] == 0 and args[20] == 68 and dX.dtype is B and dW.dtype is torch.float32
    lm._lib.calls.clear()
    assert lm.cross_entropy_backward(g, X, W, y, lse, need_dx=False)[0] is None and launched(lm)[0][1][15] is None
    # (up to 16 rows nothing is asked for a workspace)
    lm._lib.calls.clear()
    lm.linear(Tensor(16, 64, dtype=B), P)
    assert [c[0] for c in lm._lib.calls] == ["ozimmu_lm_linear_way"] and lm._lib.calls[0][1][16] is None


def test_a_gradient_that_would_be_lost_is_refused(lm):
    P, y, v = packed(lm), Tensor(20, dtype=I64), Tensor(20)
    t = lambda rows, grad: Tensor(rows, 64, dtype=B, requires_grad=grad)  # noqa: E731
    calls = [lambda: lm.linear(t(20, True), P), lambda: lm.cross_entropy(t(20, True), t(100, False), y), lambda: lm.cross_entropy(t(20, False), t(100, True), y),
             lambda: lm.cross_entropy_backward(v, t(20, True), t(100, False), y, v), lambda: lm.cross_entropy_backward(v, t(20, False), t(100, True), y, v),
             lambda: lm.cross_entropy_backward(Tensor(20, requires_grad=True), t(20, False), t(100, False), y, v)]
    for call in calls:
        lm._lib.calls.clear()
        with pytest.raises(ValueError, match="requires a gradient"):
            call()
        assert launched(lm) == []
        with torch.no_grad():
            call()
        assert len(launched(lm)) == 1
    lm.quantize(Tensor(4, 64, requires_grad=True))     # (no tensor comes of it)


def test_tensors_on_another_device_are_refused(lm, monkeypatch):
    from paper_2409_13313_amd import mx
    monkeypatch.setattr(mx, "_several_devices", True)
    calls = {"quantize": (1, lambda at: lm.quantize(Tensor(4, 64, at=at[0]))),
             "dequantize": (2, lambda at: lm.dequantize(packed(lm, at=at[0]), out=Tensor(32, 64, at=at[1]))),
             "pack": (3, lambda at: lm.pack(Tensor(4, 32, dtype=U8, at=at[0]), Tensor(4, 1, dtype=B, at=at[1]), Tensor(4, 1, dtype=U8, at=at[2]))),
             "unpack": (1, lambda at: lm.unpack(packed(lm, at=at[0]))),
             "linear": (4, lambda at: lm.linear(Tensor(20, 64, dtype=B, at=at[0]), packed(lm, at=at[1]), D=Tensor(20, 32, dtype=B, at=at[2]),
                                                workspace=Tensor(4096, dtype=U8, at=at[3]))),
             "loss": (6, lambda at: lm.cross_entropy(Tensor(20, 64, dtype=B, at=at[0]), Tensor(9, 64, dtype=B, at=at[1]), Tensor(20, dtype=I64, at=at[2]),
                                                     loss=Tensor(20, at=at[3]), lse=Tensor(20, at=at[4]), workspace=Tensor(4096, dtype=U8, at=at[5]))),
             "gradient": (8, lambda at: lm.cross_entropy_backward(Tensor(20, at=at[0]), Tensor(20, 64, dtype=B, at=at[1]), Tensor(9, 64, dtype=B, at=at[2]),
                                                                  Tensor(20, dtype=I64, at=at[3]), Tensor(20, at=at[4]), dX=Tensor(20, 64, at=at[5]),
                                                                  dW=Tensor(9, 64, at=at[6]), workspace=Tensor(4096, dtype=U8, at=at[7])))}
    for name, (count, call) in calls.items():
        lm._lib.calls.clear()
        call([1] * count)
        assert len(launched(lm)) == 1, name
        for i in range(count):
            lm._lib.calls.clear()
            with pytest.raises(ValueError, match="current device"):
                call([1] * i + [0] + [1] * (count - i - 1))
            assert launched(lm) == [], (name, i)
