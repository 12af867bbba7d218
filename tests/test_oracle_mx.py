"""The oracle of the microscaled 4-bit form against values worked out by hand."""
import numpy as np
import pytest

from oracle import mx as ref


def one(values):
    codes, scales = ref.quantize(np.array([values + [0.0] * (32 - len(values))]))
    return codes[0, :len(values)].tolist(), int(scales[0, 0])


def test_ties_go_to_the_even_code_and_the_largest_saturate():
    # amax 4 .. 7.99: scale 2^0 (byte 127)
    x = [4.0, 0.25, 0.26, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 5.01, 7.0, 7.99, -0.25, -0.75, 0.24]
    assert one(x) == ([6, 0, 1, 2, 2, 4, 4, 6, 6, 7, 7, 7, 8, 10, 0], 127)


@pytest.mark.parametrize("amax,byte", [(1.0, 125), (6.0, 127), (8.0, 128), (7.999, 127), (0.0, 0), (2.0 ** -126, 0),
                                       (2.0 ** -125, 0), (2.0 ** -124, 1), (2.0 ** -140, 0), (2.0 ** 127 * 1.99, 252)])
def test_scale_bytes(amax, byte):
    assert one([amax])[1] == byte


@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan])
def test_a_block_without_finite_values_is_nan(bad):
    X = np.ones((2, 70))
    X[1, 40] = bad
    q = ref.read_back(X)
    assert np.isnan(q[1, 32:64]).all() and np.isfinite(q[0]).all() and (q[1, :32] == 1).all() and (q[1, 64:] == 1).all()


def test_read_back_is_a_fixed_point_and_near():
    rng = np.random.default_rng(3)
    X = rng.standard_normal((5, 100)) * np.exp(rng.standard_normal((5, 100)))
    q = ref.read_back(X)
    assert np.array_equal(ref.read_back(q), q)
    big = np.abs(np.pad(X, ((0, 0), (0, 28))).reshape(5, 4, 32)).max(axis=2)
    # steps of 2 at the top: at most a quarter of amax away (saturation from just below 8 to 6)
    assert (np.abs(q - X) <= np.repeat(big, 32, axis=1)[:, :100] * 0.25 + 1e-12).all()


def test_bytes():
    codes = np.arange(32, dtype=np.uint8).reshape(1, 32) % 16
    assert np.array_equal(ref.codes_of(ref.bytes_of(codes)), codes) and ref.bytes_of(codes)[0, 0] == 0x10
