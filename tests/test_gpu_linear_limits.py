"""Gradients behind pre-activations that 16 bits do not hold: Z is kept as an infinity where Y, from the float32 sum, is the
activation's value; the slopes there are 0 or 1."""
import numpy as np
import pytest

from tests.dense_util import rounded
from tests.test_gpu_linear import FLAG, forward, gradients
from oracle import dense_oracle as orc

pytestmark = pytest.mark.gpu

ENDS = {"relu": (0.0, 1.0), "gelu": (0.0, 1.0), "gelu_tanh": (0.0, 1.0), "silu": (0.0, 1.0)}


@pytest.mark.parametrize("name", orc.ACTS[1:])
@pytest.mark.parametrize("N", [1, 9, 64, 200, 1100])  # 8, 64 and 256 threads a row
def test_a_step_whose_pre_activations_leave_f16(name, N):
    import paper_2407_20496_amd as hinm
    K = 16
    far = np.array([-1.0, 1.0, -1.0, 1.0, 0.0, 0.0, 1.0])  # rows with sums of -+ 70000, of 0, and an ordinary one
    W = np.zeros((len(far), K))
    W[:4, 0] = 35008 * far[:4]
    W[5, 1], W[6, 2] = 2.0, 0.5
    X = np.zeros((K, N))
    X[0], X[1], X[2] = 2, 0, 1
    X[5] = np.arange(N) % 5 - 2  # of no row's weight
    y, z, _, _ = forward(hinm, W, X, "f16", keep=True, flags=FLAG[name])
    kept = z.f64()
    assert np.isneginf(kept[[0, 2]]).all() and np.isposinf(kept[[1, 3]]).all()
    assert (y.f64()[[0, 2]] == 0).all() and np.isposinf(y.f64()[[1, 3]]).all()
    dY = np.tile(np.array([1.0, 2.0, -3.0, -1.0, 2.0, 1.0, 4.0])[:, None], (1, N))
    dx, dw, db = gradients(hinm, np.where(np.abs(W) > 100, np.sign(W), W), X, kept, dY, "f16", name)
    low, high = ENDS[name]
    slope = np.empty((len(far), N))
    slope[[0, 2]], slope[[1, 3]] = low, high
    slope[4:] = orc.slope(kept[4:], name)
    dZ = dY * slope
    Ws = np.where(np.abs(W) > 100, np.sign(W), W)
    # at most one rounding of dZ, one of the result, and the ordinary rows' slopes (2^-19 relative to 1 + |z|)
    near = lambda got, want, sums: (np.abs(got - want) <= (2.0 ** -11 * 2 + 2.0 ** -18) * sums + 2.0 ** -24).all()
    assert near(dx.f64(), Ws.T @ dZ, np.abs(Ws).T @ np.abs(dY)) and near(dw.f64(), dZ @ X.T, np.abs(dY) @ np.abs(X).T)
    assert near(db, dZ.sum(1), np.abs(dY).sum(1))
    # the rows far out are exact: integers times 0 or 1
    exact = rounded(dZ @ X.T, "f16")
    assert np.array_equal(dw.f64()[:4], exact[:4]) and np.array_equal(db[:4], dZ.sum(1)[:4])


@pytest.mark.parametrize("name", orc.ACTS[1:])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_a_pre_activation_that_is_no_number_stays_one(name, dtype):
    """In its own row of dW and of the bias, its own column of dX; infinities beside it have their slopes."""
    import paper_2407_20496_amd as hinm
    M, K, N = 6, 8, 24
    Z = np.ones((M, N))
    Z[1, 3], Z[2], Z[3] = np.nan, -np.inf, np.inf
    dx, dw, db = gradients(hinm, np.ones((M, K)), np.ones((K, N)), Z, np.ones((M, N)), dtype, name)
    assert np.isnan(db[1]) and np.isnan(dw.f64()[1]).all() and np.isnan(dx.f64()[:, 3]).all()
    assert np.isfinite(np.delete(db, 1)).all() and np.isfinite(np.delete(dw.f64(), 1, 0)).all() and np.isfinite(np.delete(dx.f64(), 3, 1)).all()
    assert db[2] == 0 and db[3] == N and (dw.f64()[2] == 0).all() and (dw.f64()[3] == N).all()
