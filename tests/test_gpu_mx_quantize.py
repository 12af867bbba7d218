"""Quantisation to the microscaled 4-bit form, reading back and the plain layout against the definition in 64 bits: equal codes, equal
scale bytes, equal values."""
import numpy as np
import pytest

from oracle import mx as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZES = [(1, 1), (1, 4096), (2, 31), (3, 32), (5, 33), (16, 128), (17, 127), (64, 129), (65, 256), (255, 160), (257, 513), (300, 1001)]


@pytest.fixture(scope="module")
def mx():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU: the HIP path has no CPU fallback")
    from paper_2409_13313_amd import mx
    return mx


def matrix(rows, n, kind, seed, spread=2.0, pad=0):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, n + pad)) * np.exp(spread * rng.standard_normal((rows, n + pad)))
    x[rng.random((rows, n + pad)) < 0.05] = 0.0
    if rows > 3:
        x[rows // 2] = 0.0                      # a row without anything
    return torch.from_numpy(x).to(TYPES[kind]).cuda()[:, :n]


def same(mx, packed, X64):
    """The packed matrix is X64 quantised: codes where the block is finite, scale bytes everywhere."""
    codes, scales = (t.cpu().numpy() for t in mx.unpack(packed))
    want_codes, want_scales = ref.quantize(X64)
    assert np.array_equal(scales, want_scales)
    fine = np.repeat(want_scales != 255, 32, axis=1)
    assert np.array_equal(ref.codes_of(codes)[fine], want_codes[fine])


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("rows,n", SIZES)
def test_both_ways(mx, kind, rows, n):
    for pad in (0, 1, 8):
        X = matrix(rows, n, kind, rows * 7 + n, pad=pad)
        X64 = X.double().cpu().numpy()
        by_row, by_col = mx.quantize(X, rows=True, cols=True)
        same(mx, by_row, X64)
        same(mx, by_col, X64.T)
        only_row, none = mx.quantize(X)
        assert none is None
        same(mx, only_row, X64)
        none, only_col = mx.quantize(X, rows=False, cols=True)
        assert none is None
        same(mx, only_col, X64.T)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("rows,n", SIZES)
def test_reading_back(mx, kind, rows, n):
    X = matrix(rows, n, kind, rows + n)
    by_row, by_col = mx.quantize(X, rows=True, cols=True)
    want, want_t = ref.read_back(X.double().cpu().numpy()), ref.read_back(X.double().cpu().numpy().T)
    for out_kind, t in TYPES.items():
        rounded = torch.from_numpy(want).to(t)
        assert torch.equal(mx.dequantize(by_row, t).cpu(), rounded), out_kind
        assert torch.equal(mx.dequantize(by_col, t).cpu(), torch.from_numpy(want_t).to(t)), out_kind
        big = torch.full((rows, n + 3), 7.0, dtype=t, device="cuda")
        mx.dequantize(by_row, t, out=big[:, 1:n + 1])
        assert torch.equal(big[:, 1:n + 1].cpu(), rounded) and (big[:, 0] == 7).all() and (big[:, n + 1:] == 7).all()


@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_every_value_of_16_bits(mx, kind):
    """Each finite value beside a largest one up to twelve binades above it, and as the largest itself."""
    t = TYPES[kind]
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16)
    x = bits.view(t)
    x = x[torch.isfinite(x)]
    for up in (None, 0, 1, 2, 3, 4, 12):
        y = torch.zeros((x.numel(), 32), dtype=t)
        y[:, 5] = x
        if up is not None:
            y[:, 20] = (x.double().abs() * 2.0 ** up).clamp(max=torch.finfo(t).max).to(t)
        got, _ = mx.quantize(y.cuda())
        same(mx, got, y.double().numpy())
        assert torch.equal(mx.dequantize(got, torch.float32).cpu().double(), torch.from_numpy(ref.read_back(y.double().numpy())))


def test_32_bit_values_at_the_edges(mx):
    """Around every rounding point and at both ends of the exponents, subnormal numbers among them."""
    points = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0], dtype=np.float32)
    near = np.concatenate([points, np.nextafter(points, np.float32(0)), np.nextafter(points, np.float32(99)), -points])
    rows = []
    for e in list(range(-149, -100)) + [-60, -1, 0, 1, 60] + list(range(118, 126)):
        row = np.zeros(32, dtype=np.float32)
        with np.errstate(all="ignore"):
            scaled = np.ldexp(near, e).astype(np.float32)
            top = np.ldexp(np.float32(4.0), e).astype(np.float32)
        for start in range(0, len(near), 31):
            row = np.zeros(32, dtype=np.float32)
            part = scaled[start:start + 31]
            row[:len(part)], row[31] = part, top
            rows.append(row)
    rows.append(np.full(32, np.finfo(np.float32).max, dtype=np.float32))
    X = np.stack(rows)
    assert np.isfinite(X).all()
    got, _ = mx.quantize(torch.from_numpy(X).cuda())
    same(mx, got, X.astype(np.float64))
    _, got = mx.quantize(torch.from_numpy(np.ascontiguousarray(X.T)).cuda(), rows=False, cols=True)
    same(mx, got, X.astype(np.float64))


@pytest.mark.parametrize("kind", list(TYPES))
def test_blocks_that_are_not_finite(mx, kind):
    X = matrix(70, 200, kind, 5)
    X[3, 40], X[20, 199], X[69, 0] = float("inf"), float("nan"), float("-inf")
    X64 = X.double().cpu().numpy()
    by_row, by_col = mx.quantize(X, rows=True, cols=True)
    same(mx, by_row, X64)
    same(mx, by_col, X64.T)
    for t in TYPES.values():
        assert torch.equal(torch.isnan(mx.dequantize(by_row, t)).cpu(), torch.from_numpy(np.isnan(ref.read_back(X64))))


def test_plain_layout(mx):
    rng = np.random.default_rng(9)
    for rows, n in ((1, 1), (3, 40), (64, 128), (300, 1001)):
        blocks = -(-n // 32)
        codes = rng.integers(0, 256, (rows, blocks * 16 + 5), dtype=np.uint8)
        scales = rng.integers(0, 256, (rows, blocks + 2), dtype=np.uint8)
        dc, ds = torch.from_numpy(codes).cuda()[:, 3:3 + blocks * 16], torch.from_numpy(scales).cuda()[:, 1:1 + blocks]
        P = mx.pack(dc, ds, n)
        got_codes, got_scales = (t.cpu().numpy() for t in mx.unpack(P))
        want = ref.codes_of(codes[:, 3:3 + blocks * 16])
        want[:, n:] = 0
        assert np.array_equal(ref.codes_of(got_codes), want) and np.array_equal(got_scales, scales[:, 1:1 + blocks])
        with np.errstate(over="ignore"):   # (6 x 2^127 is infinite in 32 bits)
            values = ref.values(want, got_scales, n).astype(np.float32)
        assert np.array_equal(mx.dequantize(P).cpu().numpy(), values, equal_nan=True)


@pytest.mark.parametrize("kind", list(TYPES))
def test_every_code_with_every_scale(mx, kind):
    """Values that the type cannot hold are rounded once, to infinity and to subnormal numbers too."""
    codes = np.tile(np.arange(32, dtype=np.uint8) % 16, (256, 1))
    scales = np.arange(256, dtype=np.uint8).reshape(256, 1)
    P = mx.pack(torch.from_numpy(ref.bytes_of(codes)).cuda(), torch.from_numpy(scales).cuda())
    want = torch.from_numpy(ref.values(codes, scales, 32)).to(TYPES[kind])
    got = mx.dequantize(P, TYPES[kind]).cpu()
    fine = ~torch.isnan(want)
    assert torch.equal(torch.isnan(got), ~fine) and torch.equal(got[fine], want[fine])


def test_rows_far_behind_2_32_bytes(mx):
    """A view whose last row begins behind 4 GiB."""
    ld = (1 << 31) + 8
    flat = torch.zeros(2 * ld + 64, dtype=torch.bfloat16, device="cuda")
    X = torch.as_strided(flat, (3, 64), (ld, 1))
    X.copy_(matrix(3, 64, "bf16", 4))
    by_row, by_col = mx.quantize(X, rows=True, cols=True)
    X64 = X.double().cpu().numpy()
    same(mx, by_row, X64)
    same(mx, by_col, X64.T)
    X.zero_()
    mx.dequantize(by_row, torch.bfloat16, out=X)
    assert np.array_equal(X.double().cpu().numpy(), ref.read_back(X64))


def test_nothing_to_do(mx):
    for rows, n in ((0, 64), (5, 0)):
        X = torch.empty((rows, n), device="cuda")
        by_row, by_col = mx.quantize(X, rows=True, cols=True)
        assert by_row.shape == (rows, n) and by_col.shape == (n, rows)
        assert mx.dequantize(by_row).shape == (rows, n)
        codes, scales = mx.unpack(by_row)
        assert mx.pack(codes, scales, n).shape == (rows, n)


def test_another_stream(mx):
    X = matrix(300, 700, "bf16", 8)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        by_row, by_col = mx.quantize(X, rows=True, cols=True)
    torch.cuda.current_stream().wait_stream(s)
    same(mx, by_row, X.double().cpu().numpy())
    same(mx, by_col, X.double().cpu().numpy().T)
