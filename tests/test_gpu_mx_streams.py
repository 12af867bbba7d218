"""Every microscaled 4-bit operator on another stream than the one its operands were made on, behind long work of that stream that the operands wait for:
work on any other stream would find the operands of before, or NaN where results are."""
import pytest

from test_gpu_mx_product import matrix, mx  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def test_all_of_them_behind_long_work(mx):  # noqa: F811
    m, n, p = 200, 3000, 400
    new = {"X": matrix(m, n, "bf16", 1), "W": matrix(p, n, "bf16", 2), "G": matrix(m, p, "bf16", 3)}
    held = {k: torch.full_like(v, 1.0) for k, v in new.items()}
    out = {"Y": (m, p), "few": (16, p), "dX": (m, n), "dW": (p, n), "gemm": (m, p), "back": (p, n), "again": (n, p)}
    out = {k: torch.empty(s, device="cuda") for k, s in out.items()}
    ws = mx.alloc_workspace(m, n, p, backward=True)

    def step():
        X, W, G = (held[k] for k in ("X", "W", "G"))
        by_row, by_col = mx.quantize(W, rows=True, cols=True)
        mx.linear(X, by_row, D=out["Y"], workspace=ws)
        mx.linear(X[:16], by_row, D=out["few"])
        mx.linear_backward(G, X, by_col, dX=out["dX"], dW=out["dW"], workspace=ws)
        mx.gemm(mx.quantize(X)[0], by_row, D=out["gemm"])
        mx.dequantize(by_row, out=out["back"])
        mx.dequantize(mx.pack(*mx.unpack(by_col), p), out=out["again"])

    def clear():
        for t in out.values():
            t.fill_(float("nan"))

    step()
    old = {k: t.clone() for k, t in out.items()}
    for k, t in new.items():
        held[k].copy_(t)
    step()
    want = {k: t.clone() for k, t in out.items()}
    assert all(not torch.equal(old[k], want[k]) and torch.isfinite(want[k]).all() for k in out)
    big = torch.randn((8192, 8192), device="cuda").bfloat16()
    stream = torch.cuda.Stream()
    for _ in range(3):
        clear()
        for t in held.values():
            t.fill_(1.0)
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            for _ in range(8):
                big = torch.mm(big, big).mul_(2.0 ** -7)
            for k, t in new.items():
                held[k].copy_(t)
            step()
        torch.cuda.current_stream().wait_stream(stream)
        for k, t in out.items():
            assert torch.equal(t, want[k]), k
    torch.cuda.synchronize()
