"""Layer norm of tokens whose mean is all that they hold: deviations of zero, at every size of values and in every form."""
import numpy as np
import pytest

from tests.dense_util import Matrix, result, workspace

pytestmark = pytest.mark.gpu

# vectors of 512 and 1024 threads, one and two rounds of them; columns held; strips
VECTORS = [(4095, 1), (8191, 1), (8193, 1), (9001, 1), (12287, 1), (16383, 1), (16384, 1)]
SHAPES = VECTORS + [(1, 1), (100, 9), (1000, 7), (1024, 130), (2047, 8), (4095, 5), (5000, 63), (3001, 200), (16383, 9)]


def _constant(K, N, dtype, value, eps=1e-5):
    import torch
    import paper_2407_20496_amd as hinm
    x, u = Matrix(K, N, dtype, values=np.full((K, N), value)), result(K, N, dtype)
    b = torch.full((K,), 0.5, device="cuda:0")
    w = torch.full((K,), 3.0, device="cuda:0")
    mean, rstd = (torch.full((N,), 77.0, device="cuda:0") for _ in range(2))
    hinm.hinm_layer_norm(K, N, dtype, eps, x.data, x.ld, w, b, u.data, u.ld, mean, rstd, *workspace(hinm.hinm_layer_norm_workspace(K, N)))
    torch.cuda.synchronize()
    return u.f64(), mean.double().cpu().numpy(), rstd.double().cpu().numpy()


@pytest.mark.parametrize("K,N", SHAPES)
@pytest.mark.parametrize("dtype,value", [("f16", 65504.0), ("f16", -2047.0 * 2 ** -7), ("bf16", 255.0 * 2 ** 12), ("bf16", 3.0)])
def test_equal_channels(K, N, dtype, value):
    """K equal values have themselves as their mean, exactly (their sum needs 11 + 14 bits of float32's 24): deviations are
    zero, so the result is b however small eps is beside the values."""
    u, mean, rstd = _constant(K, N, dtype, value)
    assert (mean == value).all()
    assert (u == 0.5).all()
    assert np.allclose(rstd, 1 / np.sqrt(1e-5), rtol=2.0 ** -21, atol=0)


@pytest.mark.parametrize("K,N", SHAPES)
@pytest.mark.parametrize("value", [255.0 * 2 ** 120, -(2.0 ** 127), 2.0 ** 112])
def test_equal_channels_whose_sum_leaves_float32(K, N, value):
    u, mean, rstd = _constant(K, N, "bf16", value)
    assert (mean == value).all() and (u == 0.5).all()
    assert np.allclose(rstd, 1 / np.sqrt(1e-5), rtol=2.0 ** -21, atol=0)


@pytest.mark.parametrize("K", [k for k, _ in VECTORS])
def test_one_channel_of_a_token_apart(K):
    """One value a step beside the rest, far from zero: the smallest spread that 16 bits have."""
    import torch
    import paper_2407_20496_amd as hinm
    from oracle import dense_oracle as orc
    x = np.full((K, 1), 65472.0)
    x[K // 3] = 65504.0
    m, u = Matrix(K, 1, "f16", values=x), result(K, 1, "f16")
    mean, rstd = (torch.full((1,), 77.0, device="cuda:0") for _ in range(2))
    hinm.hinm_layer_norm(K, 1, "f16", 0.0, m.data, m.ld, None, None, u.data, u.ld, mean, rstd, *workspace(hinm.hinm_layer_norm_workspace(K, 1)))
    torch.cuda.synchronize()
    want, wm, wr = orc.layer_norm(x, None, None, 0.0)
    # deviations of 32 and 32 / K.  x less the rounded mean is exact; its own mean is off by some 16 roundings of 32 / K at most, the
    # squares' sum by as many; then three roundings and one to the type
    assert abs(mean.item() - wm[0]) <= 2.0 ** -24 * wm[0] + 2.0 ** -8
    assert abs(rstd.item() / wr[0] - 1) <= 2.0 ** -18
    off = 2.0 ** -18 * np.abs(want) + 2.0 ** -19 * 32 / K * wr[0]
    assert (np.abs(u.f64() - want) <= 2.0 ** -11 * np.abs(want) + off + 2.0 ** -24).all()
