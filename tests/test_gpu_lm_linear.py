"""The linear layer with 4-bit weights against products in 64 bits, in every way it can be run.

Bounds.  Straight from the codes, a group's sum is that of x (128 + q) in BF16 (magnitudes up to 143 |x|) or of x (q - zero) in FP16 (up to 15 |x|),
exact products; it passes through at most 6 roundings for each 32 elements of the group, and 4 more to the total; the total through at most one for each
group and 40 where waves, splits and launches meet, at magnitudes up to 15 scale |x|.  An FP32 rounding counts 2^-23 (the matrix cores may
truncate).  Weights read back in 16 bits are off by half a step of the type each.  The result is rounded once to its type, by half a step.
That bound is for the worst case; for sums of many independent roundings the norm of the error stays below one and a half half steps, which is asked for too."""
import numpy as np
import pytest

from oracle import lm as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 2.0 ** -126, "bf16": 2.0 ** -126, "f16": 2.0 ** -24}
WAYS = ("direct", "shared", "tile")
FORMS = [(32, True, "f16"), (64, False, "bf16"), (128, True, "bf16"), (128, False, "f16")]
# one row and many, sizes around the edges of fragments, blocks and tiles, rows that end anywhere, few and many of each
SHAPES = [(1, 1, 1), (1, 4096, 300), (2, 33, 17), (3, 8, 1000), (4, 129, 31), (5, 1000, 4100), (16, 520, 333), (17, 128, 16), (31, 2051, 200),
          (33, 640, 129), (64, 127, 255), (65, 3000, 70), (128, 256, 512), (133, 2051, 1283), (257, 136, 300), (300, 1000, 1000), (1100, 520, 900)]


@pytest.fixture(scope="module")
def lm():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU: the HIP path has no CPU fallback")
    from paper_2409_13313_amd import lm
    return lm


def weights(lm, p, n, group, zeros, scale, seed):
    """Packed weights and their values in 64 bits."""
    rng = np.random.default_rng(seed)
    groups = -(-n // group)
    codes = rng.integers(0, 16, (p, n)).astype(np.uint8)
    s = torch.from_numpy(np.exp(rng.uniform(-6, -4, (p, groups)))).to(TYPES[scale])
    z = rng.integers(0, 16, (p, groups)).astype(np.uint8) if zeros else None
    P = lm.pack(torch.from_numpy(ref.bytes_of(codes)).cuda(), s.cuda(), None if z is None else torch.from_numpy(z).cuda(), n=n, group=group)
    W = ref.values(codes, s.float().numpy(), np.full((p, groups), 8) if z is None else z, group)
    return P, torch.from_numpy(W).cuda(), torch.from_numpy(np.repeat(s.double().numpy(), group, axis=1)[:, :n]).cuda()


def rows(m, n, kind, seed, pad=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn((m, n + pad), device="cuda", generator=gen).to(TYPES[kind])[:, :n]


def bound(X, W, S, kind, way, group):
    """Of the FP32 sums: elementwise."""
    x, n = X.double().abs(), X.shape[1]
    if way == "tile":
        return HALF[kind] * (x @ W.abs().t()) + (6 * n / 32 + 40) * 2.0 ** -23 * (x @ W.abs().t())
    held = 143 if kind == "bf16" else 15
    return 2.0 ** -23 * ((6 * group / 32 + 4) * held + (n / group + 40) * 15) * (x @ S.t())


def check(got, want, off_sums, kind, what):
    off, got = (got.double() - want).abs(), got.double()
    limit = off_sums + HALF[kind] * (want.abs() + off_sums) + TINY[kind]
    assert (off <= limit).all(), f"{what}: {(off / limit).max().item():.3g} of the bound"
    if want.numel() >= 1000 and kind != "f32":
        assert off.norm() <= 1.5 * HALF[kind] * want.norm(), f"{what}: {(off.norm() / want.norm()).item():.3g}"


@pytest.mark.parametrize("m,n,p", SHAPES)
@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_every_way(lm, m, n, p, kind):
    for group, zeros, scale in FORMS:
        P, W, S = weights(lm, p, n, group, zeros, scale, m + n + p)
        for pad in (0, 1):
            X = rows(m, n, kind, n, pad)
            want = X.double() @ W.t()
            for way in WAYS:
                print(f"linear {m} x {n} x {p} {kind} group {group} zeros {zeros} {scale} {way}", flush=True)
                b = bound(X, W, S, kind, way, group)
                got = lm.linear(X, P, way=way)
                assert got.dtype is TYPES[kind]
                check(got, want, b, kind, f"{way} {group}")
                assert torch.equal(got, lm.linear(X, P, way=way))    # (the same call, the same bits)
        b = torch.maximum(bound(X, W, S, kind, "direct", group), bound(X, W, S, kind, "tile", group))
        check(lm.linear(X, P), want, b, kind, "as chosen")


@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("out", list(TYPES))
def test_alpha_beta_and_outputs_inside_others(lm, way, out):
    for m, n, p in ((3, 200, 100), (37, 1001, 333), (140, 264, 515)):
        P, W, S = weights(lm, p, n, 64, True, "f16", 3)
        X = rows(m, n, "bf16", 5)
        big = torch.randn((m + 1, p + 5), device="cuda").to(TYPES[out])
        before = big.clone()
        alpha, beta = -0.75, 0.5
        got = lm.linear(X, P, alpha=alpha, beta=beta, D=big[:m, 3:p + 3], way=way)
        assert got.data_ptr() == big[:m, 3:].data_ptr()
        want = alpha * (X.double() @ W.t()) + beta * before[:m, 3:p + 3].double()
        b = bound(X, W, S, "bf16", way, 64) + 2.0 ** -22 * (want.abs() + before[:m, 3:p + 3].double().abs() + (X.double() @ W.t()).abs())
        off = (got.double() - want).abs()
        assert (off <= b + HALF[out] * (want.abs() + b) + TINY[out]).all(), (m, n, p)
        changed = big.clone()
        changed[:m, 3:p + 3] = before[:m, 3:p + 3]
        assert torch.equal(changed, before)
        # beta 0: what was there is not read
        lm.linear(X, P, D=big[:m, 3:p + 3].fill_(float("nan")), way=way)
        assert torch.isfinite(big[:m, 3:p + 3]).all()


@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_what_is_not_finite_stays_in_its_row_and_its_column(lm, way, kind):
    """Packed weights in memory full of 0xff (padding rows of NaN scales), X and D inside others full of NaN, rows of X with NaN and infinities, a group
    whose scale is NaN."""
    for m, n, p, group in ((2, 77, 21, 32), (40, 300, 129, 64), (133, 1001, 270, 128)):
        print(f"{way} {kind} {m} x {n} x {p}", flush=True)
        gen = torch.Generator(device="cuda").manual_seed(1)
        W0 = torch.randn((p, n), device="cuda", generator=gen)
        W0[p // 2, n // 2] = float("nan")
        P = lm.Packed(torch.full((lm.packed_bytes(p, n, group, True),), 255, dtype=torch.uint8, device="cuda"), p, n, group, True, torch.float16)
        assert lm._lib.ozimmu_lm_quantize(0, p, n, W0.data_ptr(), n, group, 1, 2, P.data.data_ptr(), torch.cuda.current_stream().cuda_stream) == 0
        big = torch.full((m + 2, n + 9), float("nan"), device="cuda", dtype=TYPES[kind])
        big[1:m + 1, 5:n + 5] = torch.randn((m, n), device="cuda", generator=gen).to(TYPES[kind])
        X = big[1:m + 1, 5:n + 5]
        X[0, n - 1] = float("nan")
        X[m - 1, 0] = float("inf")
        got = lm.linear(X, P, way=way).float()
        fine = torch.isfinite(got)
        assert not fine[0].any() and not fine[m - 1].any() and not fine[:, p // 2].any()
        keep_rows, keep_cols = torch.arange(m, device="cuda"), torch.arange(p, device="cuda") != p // 2
        keep_rows = (keep_rows > 0) & (keep_rows < m - 1)
        assert fine[keep_rows][:, keep_cols].all()


def test_no_rows_and_no_columns(lm):
    P, _, _ = weights(lm, 20, 64, 32, False, "f16", 1)
    assert lm.linear(rows(0, 64, "bf16", 1), P).shape == (0, 20)
    none = lm.quantize(torch.empty((0, 64), device="cuda"))
    assert lm.linear(rows(3, 64, "bf16", 1), none).shape == (3, 0)
    assert lm.dequantize(none).shape == (0, 64) and lm.unpack(none)[0].shape == (0, 32)


def test_a_workspace_of_the_users_and_one_too_small(lm):
    P, W, S = weights(lm, 300, 1001, 64, True, "f16", 1)
    X = rows(500, 1001, "f16", 2)
    from paper_2409_13313_amd.ozimmu import OzimmuError
    for way in ("shared", "tile"):
        need = lm.linear_workspace_bytes(500, 1001, 300, way)
        room = torch.full((need + 256,), 255, dtype=torch.uint8, device="cuda")
        got = lm.linear(X, P, workspace=room[:need], way=way)
        assert (room[need:] == 255).all() and torch.equal(got, lm.linear(X, P, way=way))
        with pytest.raises(OzimmuError):
            lm.linear(X, P, workspace=room[:need - 256], way=way)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_pieces_of_weights_read_back(lm, kind):
    """More weights than are read back at a time: 2^27 bytes, 8192 rows of 8192."""
    m, n, p = 130, 8192, 8300
    W0 = (torch.randn((p, n), device="cuda") * 0.02).to(TYPES[kind])
    P = lm.quantize(W0)
    X = rows(m, n, kind, 3)
    W = lm.dequantize(P).double()
    got = lm.linear(X, P, way="tile")
    want = X.double() @ W.t()
    off = (got.double() - want).norm() / want.norm()
    assert off <= 1.5 * HALF[kind]
    assert torch.equal(got[:, 8192:], lm.linear(X, lm.quantize(W0[8192:]), way="tile"))


# few rows through weights of many rows, in each way they are shared out, and of more than 256 MB, which are read past the caches
@pytest.mark.parametrize("m,n,p", [(2, 264, 40000), (3, 136, 70001), (9, 264, 9000), (9, 136, 20000), (13, 264, 70001), (1, 4100, 131101), (11, 4100, 131101),
                                   (16, 33100, 16373)])
@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_few_rows_of_wide_layers(lm, m, n, p, kind):
    gen = torch.Generator(device="cuda").manual_seed(n)
    for group, zeros, scale in FORMS[:3] if n * p < 1 << 26 else FORMS[2:3]:
        P = lm.quantize(torch.randn((p, n), device="cuda", generator=gen) * 0.02, group=group, zeros=zeros, scale_type=TYPES[scale])
        W = lm.dequantize(P, torch.float32).double()   # (exact: a scale of 11 bits times at most 15)
        S = lm.unpack(P)[1].double().repeat_interleave(group, dim=1)[:, :n]
        X = rows(m, n, kind, n, 1)
        got = lm.linear(X, P, D=torch.empty((m, p), device="cuda", dtype=torch.float32))
        check(got, X.double() @ W.t(), bound(X, W, S, kind, "direct", group), "f32", (m, n, p, group))


@pytest.mark.parametrize("m,n,p", [(5, 8, 40), (9, 96, 300), (16, 1001, 4100), (16, 257, 17000), (13, 1030, 17000), (31, 515, 1000), (32, 129, 9000), (60, 333, 2000),
                                   (60, 264, 9000), (70, 130, 20000)])
@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_rows_that_begin_at_odd_elements_beside_nan(lm, m, n, p, kind):
    """The same numbers wherever the rows of X begin, in memory that is full of NaN elsewhere."""
    P, W, S = weights(lm, p, n, 64, True, "f16", m + n + p)
    X = rows(m, n, kind, n)

    def placed(begin, ld):
        room = torch.full((begin + m * ld,), float("nan"), device="cuda", dtype=X.dtype)
        at = room.as_strided((m, n), (ld, 1), begin)
        at.copy_(X)
        return at
    for way in ("direct", "shared"):
        want = lm.linear(placed(0, n + n % 2 + 2), P, dtype=torch.float32, way=way)
        check(want, X.double() @ W.t(), bound(X, W, S, kind, way, 64), "f32", (m, n, p, way))
        for begin, ld in ((1, n + n % 2 + 2), (0, n + 1 - n % 2), (1, n + 1 - n % 2), (1, n + 3 - n % 2)):
            assert torch.equal(lm.linear(placed(begin, ld), P, dtype=torch.float32, way=way), want), (way, begin, ld)
