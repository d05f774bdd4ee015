"""Activations in float32 results, each against its own value: the tails, where it is small, count as much as the rest."""
import numpy as np
import pytest

from tests.test_gpu_linear import FLAG, forward
from oracle import dense_oracle as orc

pytestmark = pytest.mark.gpu

STEP = 2.0 ** -24  # a rounding


def _argument(z, name):
    """Of the exponential that makes the tail, with the roundings on its way: relative, hence of the result as many of its value."""
    if name == "gelu":  # x^2, half of log2 e, their product
        return z * z / 2, 3
    if name == "silu":  # log2 e and the product with it
        return np.abs(z), 2
    # the cube's factor (three constants), x^2, the two together, times x, log2 e and the product with it
    return 2 * np.sqrt(2 / np.pi) * np.abs(z + 0.044715 * z ** 3), 8


# gelu: the fit 1.5e-7; t = 1 / (1 + 0.3 x) off by three, which the fraction takes up to 2.7 times; nine steps of a sum whose terms are 1.9
# times its value at most; four more.  The others: 1 + exp, its reciprocal, exp itself, products
REST = {"gelu": 2.0 ** -19, "silu": 2.0 ** -21, "gelu_tanh": 2.0 ** -21}
RANGE = {"gelu": (-13, 13), "silu": (-80, 80), "gelu_tanh": (-9, 20)}  # as far as the results are normal numbers


@pytest.mark.parametrize("name", REST)
@pytest.mark.parametrize("N", [1, 8, 40])  # few tokens as a vector and not, tiles
def test_tails(name, N):
    import paper_2407_20496_amd as hinm
    z = np.linspace(*RANGE[name], 4001).astype(np.float16).astype(np.float64)
    W = np.zeros((len(z), 8))
    W[:, 0] = z
    X = np.zeros((8, N))
    X[0] = 1
    got = forward(hinm, W, X, "f16", flags=FLAG[name] | 2)[0].f64()
    want = orc.act(z, name)[:, None]
    exponent, roundings = _argument(z, name)
    off = (REST[name] + roundings * STEP * exponent)[:, None]
    worst = np.max(np.abs(got - want) / np.where(want == 0, 1, np.abs(want)) / off)
    assert (np.abs(got - want) <= off * np.abs(want)).all(), worst
