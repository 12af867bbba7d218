"""The 4-bit layer of FP16 rows with BF16 scales of any magnitude, in every way it can be run, against products in 64 bits.

Bounds are those of test_gpu_lm_linear.py.  Weights read back are held times a power of two that brings the largest scale to 2^11 .. 2^12, so that each is off by 2^-11 of
itself, or by 2^-25, which is 2^-36 of the largest scale at the most."""
import pytest

torch = pytest.importorskip("torch")
from test_gpu_lm_linear import TINY, bound, lm, rows  # noqa: E402,F401

pytestmark = pytest.mark.gpu


def stored(lm, p, n, group, zeros, low, high, seed):  # noqa: F811
    """Packed weights with scales of 2^low to 2^high, and their values and scales in 64 bits."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    groups = -(-n // group)
    codes = torch.randint(0, 256, (p, -(-n // 2)), device="cuda", generator=gen, dtype=torch.uint8)
    s = (torch.rand((p, groups), device="cuda", generator=gen) + 1) * 2.0 ** torch.randint(low, high + 1, (p, groups), device="cuda", generator=gen).float()
    s = s.bfloat16()
    z = torch.randint(0, 16, (p, groups), device="cuda", generator=gen, dtype=torch.uint8) if zeros else None
    P = lm.pack(codes, s, z, n=n, group=group)
    q = torch.stack([codes & 15, codes >> 4], 2).view(p, -1)[:, :n].double()
    each = lambda t: t.double().repeat_interleave(group, 1)[:, :n]  # noqa: E731
    return P, (q - (each(z) if zeros else 8.0)) * each(s), each(s)


# X as it is, room for what the scales are scaled by beside W or behind X, in one piece or two
@pytest.mark.parametrize("m,n,p,pad", [(40, 136, 256, 0), (1, 64, 512, 0), (3, 65, 256, 0), (133, 1001, 512, 1), (700, 520, 300, 0), (700, 264, 4096, 8), (33, 77, 21, 0)])
@pytest.mark.parametrize("low,high", [(-60, -60), (-30, -26), (-20, -18), (-25, 0), (-9, -6), (0, 10), (10, 14), (40, 60)])
def test_scales_of_every_magnitude(lm, m, n, p, pad, low, high):  # noqa: F811
    for group, zeros in ((32, True), (128, False), (64, True)):
        P, W, S = stored(lm, p, n, group, zeros, low, high, m + n)
        X = rows(m, n, "f16", n, pad)
        want = X.double() @ W.t()
        for way in ("direct", "shared", "tile", "auto"):
            got = lm.linear(X, P, dtype=torch.float32, way=way)
            b = bound(X, W, S, "f16", "tile" if way == "auto" else way, group)
            if way in ("tile", "auto"):
                b = torch.maximum(b, bound(X, W, S, "f16", "direct", group)) if way == "auto" else b
                b = b + 2.0 ** -36 * S.max() * X.double().abs().sum(1, keepdim=True)
            off = (got.double() - want).abs()
            assert (off <= b + 2.0 ** -24 * (want.abs() + b) + TINY["f32"]).all(), (way, group, (off / (b + 1e-300)).max().item())
        alone = torch.full((m, p), 2.0 * float(S.max()), device="cuda")
        both = alone.clone()
        lm.linear(X, P, alpha=0.5, beta=-1.0, D=both, way="tile")
        off = (both.double() - (0.5 * want - alone.double())).abs()
        b = 0.5 * (bound(X, W, S, "f16", "tile", group) + 2.0 ** -36 * S.max() * X.double().abs().sum(1, keepdim=True))
        assert (off <= b + 2.0 ** -22 * (want.abs() + alone.double()) + TINY["f32"]).all()


def test_groups_without_a_number_and_rows_behind_the_last(lm):  # noqa: F811
    """A NaN and an infinity among the scales change their own columns alone, and what stands in padding rows nothing."""
    P, W, S = stored(lm, 300, 200, 32, False, -20, -18, 5)
    codes, scales, _ = lm.unpack(P)
    X = rows(140, 200, "f16", 1)
    want = lm.linear(X, P, dtype=torch.float32, way="tile")
    scales[7, 2], scales[50, 0] = float("nan"), float("inf")
    dirty = lm.Packed(torch.full_like(P.data, 0x7f), 300, 200, 32, False, torch.bfloat16)
    made = lm.pack(codes, scales, n=200, group=32)
    assert lm._lib.ozimmu_lm_pack(300, 200, 32, codes.data_ptr(), 100, scales.data_ptr(), 7, None, 0, dirty.data.data_ptr(), torch.cuda.current_stream().cuda_stream) == 0
    keep = torch.ones(300, dtype=torch.bool, device="cuda")
    keep[[7, 50]] = False
    for Q in (made, dirty):
        got = lm.linear(X, Q, dtype=torch.float32, way="tile")
        assert torch.isnan(got[:, 7]).all() and not torch.isfinite(got[:, 50]).any() and torch.equal(got[:, keep], want[:, keep])


def test_a_captured_layer_whose_weights_change(lm):  # noqa: F811
    """Replayed with weights of other magnitudes in the same place: what they are scaled by is found at each replay."""
    sets = [stored(lm, 300, 200, 64, True, low, high, 3)[0] for low, high in ((-3, 0), (-30, -28), (40, 41))]
    X = rows(700, 200, "f16", 1)
    P = lm.Packed(sets[0].data.clone(), 300, 200, 64, True, torch.bfloat16)
    D = torch.empty((700, 300), device="cuda")
    room = torch.empty(lm.linear_workspace_bytes(700, 200, 300, "tile"), dtype=torch.uint8, device="cuda")
    run = lambda: lm.linear(X, P, D=D, workspace=room, way="tile")  # noqa: E731
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for i in range(6):
        Q = sets[(i + 1) % 3]
        P.data.copy_(Q.data)
        room.fill_(255)
        graph.replay()
        want = lm.linear(X, Q, dtype=torch.float32, way="tile")      # (eager work between replays)
        assert torch.equal(D, want) and torch.isfinite(D).all(), i
        if i % 3 == 0:
            torch.cuda.synchronize()
