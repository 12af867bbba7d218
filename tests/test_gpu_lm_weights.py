"""4-bit weights with a scale per group: codes, scales and zero points as the definition has them, to the last bit, read back and laid out."""
import numpy as np
import pytest

from oracle import lm as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
GROUPS = (32, 64, 128)


@pytest.fixture(scope="module")
def lm():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU: the HIP path has no CPU fallback")
    from paper_2409_13313_amd import lm
    return lm


def plain(P, lm):
    """Codes (one a byte), scales and zero points (8 without) as arrays."""
    codes, scales, zeros = lm.unpack(P)
    c = codes.cpu().numpy()
    out = np.empty((P.rows, 2 * c.shape[1]), dtype=np.uint8)
    out[:, 0::2], out[:, 1::2] = c & 15, c >> 4
    if P.n % 2:
        assert (out[:, -1] == 0).all()
    s = scales.float().cpu().numpy()
    return out[:, :P.n], s, np.full(s.shape, 8, dtype=np.uint8) if zeros is None else zeros.cpu().numpy()


def same(W, lm, group, zeros, scale, what):
    P = lm.quantize(W, group=group, zeros=zeros, scale_type=TYPES[scale])
    got, want = plain(P, lm), ref.quantize(W.float().cpu().numpy(), group, zeros, scale)
    good = ~np.isnan(want[1])
    assert np.array_equal(np.isnan(got[1]), ~good) and np.array_equal(got[1][good], want[1][good]), f"{what}: scales"
    each = np.repeat(good, group, axis=1)[:, :P.n]
    assert np.array_equal(got[0][each], want[0][each]), f"{what}: {(got[0] != want[0])[each].sum()} codes"
    if zeros:
        assert np.array_equal(got[2][good], want[2][good]), f"{what}: zero points"
    return P, want


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("group", GROUPS)
@pytest.mark.parametrize("zeros", [False, True])
def test_quantisation(lm, kind, group, zeros):
    rng = np.random.default_rng(group + zeros)
    for p, n, pad in ((1, 1, 0), (1, 128, 0), (16, 128, 0), (17, 129, 3), (100, 1000, 1), (33, 31, 0), (3, 4099, 0), (257, 64, 5)):
        for scale in ("f16", "bf16"):
            print(f"quantize {p} x {n} {kind} group {group} zeros {zeros} {scale}", flush=True)
            x = rng.standard_normal((p, n + pad)) * np.exp(rng.standard_normal((p, 1)))
            x[p // 2, : n // 2] = 0.0
            W = torch.from_numpy(x).to(TYPES[kind]).cuda()[:, :n]
            P, want = same(W, lm, group, zeros, scale, f"{p} x {n}")
            v = torch.from_numpy(ref.values(*want, group)).cuda()
            for t in TYPES.values():
                # (a product of 4 and 11 bits: exact in FP32, rounded once)
                assert torch.equal(lm.dequantize(P, t), v.float().to(t))
                big = torch.full((p + 1, n + 5), 5.0, dtype=t, device="cuda")
                lm.dequantize(P, out=big[:p, 2:n + 2])
                assert torch.equal(big[:p, 2:n + 2], v.float().to(t)) and (big[:, :2] == 5).all() and (big[:, n + 2:] == 5).all() and (big[p] == 5).all()


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("zeros", [False, True])
def test_elements_half_way_between_two_codes(lm, kind, zeros):
    """Multiples of half a scale, in groups whose scale is any number of the type."""
    rng = np.random.default_rng(5)
    p = 400
    x = np.zeros((p, 128))
    s = torch.from_numpy(np.exp(rng.uniform(-4, 2, p))).to(TYPES[kind]).double().numpy()[:, None]
    x[:, :30] = (np.arange(30) - (10 if zeros else 14)) / 2 * s
    x[:, 30] = 7.5 * s[:, 0] if zeros else 7 * s[:, 0]
    W = torch.from_numpy(x).to(TYPES[kind]).cuda()
    for scale in ("f16", "bf16"):
        same(W, lm, 32, zeros, scale, "half way")


@pytest.mark.parametrize("zeros", [False, True])
def test_extremes(lm, zeros):
    rng = np.random.default_rng(9)
    for kind, spans in (("f32", (1e-45, 1e-40, 1e-38, 2.0 ** -120, 1e-30, 1e-8, 1e30, 3e38)), ("bf16", (1e-40, 1e-38, 1e-8, 1e30, 3e38)),
                        ("f16", (6e-8, 1e-6, 6e4))):
        for span in spans:
            x = rng.uniform(-1, 1, (7, 200)) * span
            W = torch.from_numpy(x).to(TYPES[kind]).cuda()
            for scale in ("f16", "bf16"):
                same(W, lm, 64, zeros, scale, f"{kind} {span}")
    for bad in (float("inf"), float("-inf"), float("nan")):
        W = torch.randn((20, 300), device="cuda")
        W[3, 130] = bad
        W[19, 299] = bad
        P, _ = same(W, lm, 128, zeros, "bf16", str(bad))
        back = lm.dequantize(P)
        assert torch.isnan(back[3, 128:256]).all() and torch.isnan(back[19, 256:]).all() and torch.isnan(back).sum() == 128 + 44


@pytest.mark.parametrize("group", GROUPS)
def test_plain_layout_there_and_back(lm, group):
    rng = np.random.default_rng(group)
    for p, n in ((1, 1), (16, 128), (17, 257), (40, 1000), (100, 77)):
        for zeros in (False, True):
            groups = -(-n // group)
            codes = rng.integers(0, 16, (p, n)).astype(np.uint8)
            data = torch.from_numpy(ref.bytes_of(codes)).cuda()
            if n % 2:
                data[:, -1] |= 0xf0                                  # (behind the end of a row: not looked at)
            scales = torch.rand((p, groups + 1), device="cuda").to(torch.float16)[:, :groups]
            z = torch.from_numpy(rng.integers(0, 16, (p, groups + 2)).astype(np.uint8)).cuda()[:, 1:groups + 1] if zeros else None
            wide = torch.full((p, data.shape[1] + 3), 255, dtype=torch.uint8, device="cuda")
            wide[:, 1:data.shape[1] + 1] = data
            P = lm.pack(wide[:, 1:data.shape[1] + 1], scales, None if z is None else z | 0x50, n=n, group=group)   # (the upper bits neither)
            got = plain(P, lm)
            assert np.array_equal(got[0], codes) and np.array_equal(got[1], scales.float().cpu().numpy())
            if zeros:
                assert np.array_equal(got[2], z.cpu().numpy())
            want = ref.values(codes, scales.float().cpu().numpy(), got[2], group)
            assert np.array_equal(lm.dequantize(P).double().cpu().numpy(), want)


def test_many_rows_of_few_elements_and_the_reverse(lm):
    """Grids that are wide one way (2^19 rows in more than one layer of the grid)."""
    for p, n in ((600000, 40), (3, 600000)):
        W = torch.randn((p, n), device="cuda", dtype=torch.float16)
        P = lm.quantize(W, group=32)
        half = lm.quantize(W[p // 2:], group=32)
        assert torch.equal(lm.dequantize(P)[p // 2:], lm.dequantize(half))
        off = (lm.dequantize(P) - W.float()).abs()
        step = torch.nn.functional.pad(W.float(), (0, -n % 32)).view(p, -1, 32).abs().amax(2) / 7 * (1 + 2.0 ** -10)
        assert (off <= step.repeat_interleave(32, 1)[:, :n] / 2 + 1e-6).all()
