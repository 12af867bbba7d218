"""The oracle of 4-bit weights and of the cross entropy against values worked out by hand, and its gradient against differences."""
import numpy as np
import pytest

from oracle import lm as ref


def test_quantisation_without_zero_points():
    # largest magnitude 7: scale 1; ties to the even code
    W = np.zeros((1, 32), dtype=np.float32)
    W[0, :9] = [7, -7, 0.5, 1.5, 2.5, -0.5, -1.5, 3.49, 0]
    q, s, z = ref.quantize(W, 32, False, "f16")
    assert s.tolist() == [[1.0]] and z.tolist() == [[8]]
    assert q[0, :9].tolist() == [15, 1, 8, 10, 10, 8, 6, 11, 8] and (q[0, 9:] == 8).all()
    assert ref.values(q, s, z, 32)[0, :3].tolist() == [7, -7, 0]


def test_quantisation_with_zero_points():
    # from -5 to 10: scale 1, zero point 5; all of one sign: zero is among the values
    W = np.array([[-5, 10, 0, 2.5, 3.5, -4.6], [3, 15, 7, 1, 2, 4]], dtype=np.float32)
    q, s, z = ref.quantize(W, 32, True, "bf16")
    assert s.tolist() == [[1.0], [1.0]] and z.tolist() == [[5], [0]]
    assert q.tolist() == [[0, 15, 5, 7, 9, 0], [3, 15, 7, 1, 2, 4]]


@pytest.mark.parametrize("zeros", [False, True])
def test_groups_of_nothing_and_of_what_is_not_finite(zeros):
    W = np.ones((3, 70), dtype=np.float32)
    W[0] = 0
    W[1, 40] = np.inf
    W[2, 69] = np.nan
    q, s, z = ref.quantize(W, 32, zeros, "f16")
    v = ref.values(q, s, z, 32)
    assert (v[0] == 0).all() and s[0].tolist() == [0, 0, 0]
    assert np.isnan(v[1, 32:64]).all() and np.isfinite(v[1, :32]).all() and np.isnan(v[2, 64:]).all()


def test_scales_that_a_type_cannot_hold():
    assert ref.to_scale(np.float32(1e6), "f16") == 65504 and ref.to_scale(np.float32(1e-9), "f16") == 0
    assert ref.to_scale(np.float32(3.4e38), "bf16") == np.float32(3.3895314e38)
    assert ref.to_scale(np.float32(1 + 2.0 ** -8), "bf16") == 1 and ref.to_scale(np.float32(1 + 3 * 2.0 ** -8), "bf16") == 1 + 2.0 ** -6


def test_loss_of_two_words():
    X, W = np.array([[1.0], [2.0], [5.0]]), np.array([[0.0], [1.0]])
    loss, lse = ref.cross_entropy(X, W, [1, 0, -100], -100)
    assert np.allclose(loss, [np.log1p(np.exp(-1)), np.log1p(np.exp(2)), 0]) and np.allclose(lse, np.log1p(np.exp([1.0, 2, 5])))
    assert np.isnan(ref.cross_entropy(X, W, [2, 0, -1], -100)[0]).tolist() == [True, False, True]


def test_gradient_against_differences():
    rng = np.random.default_rng(0)
    X, W, g = rng.standard_normal((5, 4)), rng.standard_normal((6, 4)), rng.standard_normal(5)
    y = [0, 5, -100, 2, 2]
    value = lambda X, W: (g * ref.cross_entropy(X, W, y, -100)[0]).sum()  # noqa: E731
    dX, dW = ref.backward(X, W, y, g, -100)
    h = 1e-5  # (an error of h^2 and of 2^-53 / h, both about 1e-10)
    for A, dA, f in ((X, dX, lambda A: value(A, W)), (W, dW, lambda A: value(X, A))):
        for at in np.ndindex(A.shape):
            E = np.zeros_like(A)
            E[at] = h
            assert abs((f(A + E) - f(A - E)) / (2 * h) - dA[at]) < 1e-8
    assert (dX[2] == 0).all()
