"""A block's buffers are 16-bit: layers that ask for float32 results, which take twice the memory, are refused.  On the CPU."""
import pytest
import torch

import paper_2407_20496_amd as hinm
from paper_2407_20496_amd import block as blk

K, F, N = 32, 64, 20
NOT_ONE_ACTIVATION = [hinm.OUT_F32, hinm.OUT_F32 | hinm.EPI_RELU, hinm.EPI_GELU | hinm.EPI_SILU, hinm.KERNEL_GEMV, 32, -1, 1 << 32]


def _dense(m, k, flags=0):
    """Built directly, past what dense_layer looks at."""
    return blk.DenseLayer(m, k, torch.float16, torch.zeros(m, k, dtype=torch.float16), None, flags)


def _mx4(m, k, flags=0):
    return blk.Mx4Layer(m, k, torch.float16, *blk.mx4_form(m, k, "cpu"), flags)


def _prepared(m, k, flags=0):
    return hinm.Layer(m, k, 32, k // 2, "f16", None, None, None, flags=flags)


@pytest.mark.parametrize("flags", NOT_ONE_ACTIVATION)
@pytest.mark.parametrize("where", [0, 1])
def test_dense_layers_have_one_activation_or_none(flags, where):
    shapes = [(F, K), (K, F)]
    layers = [_dense(*s, flags if i == where else 0) for i, s in enumerate(shapes)]
    with pytest.raises(ValueError):
        blk.FeedForward(layers, N, None, device="cpu")
    with pytest.raises(ValueError):
        blk.LayerNormFeedForward(layers, N, device="cpu")


@pytest.mark.parametrize("make", [_mx4, _prepared], ids=["4 bits", "prepared"])
@pytest.mark.parametrize("flags", [hinm.OUT_F32, hinm.OUT_F32 | hinm.EPI_RELU])
@pytest.mark.parametrize("where", [0, 1])
def test_compressed_layers_do_not_ask_for_float32(make, flags, where):
    layers = [make(*s, flags if i == where else 0) for i, s in enumerate([(F, K), (K, F)])]
    with pytest.raises(ValueError):
        blk.FeedForward(layers, N, None, device="cpu")


@pytest.mark.parametrize("flags", [0, hinm.EPI_RELU, hinm.EPI_GELU, hinm.EPI_GELU_TANH, hinm.EPI_SILU])
def test_activations_are_taken(flags):
    blk.FeedForward([_dense(F, K, flags), _dense(K, F, flags)], N, None, device="cpu")
    blk.LayerNormFeedForward([_dense(F, K, flags), _dense(K, F)], N, device="cpu")
    blk.FeedForward([_mx4(F, K, hinm.EPI_RELU), _mx4(K, F)], N, None, device="cpu")
