"""Limits of sizes of the 4-bit layers and norms, host side.  Every case is refused before anything is launched."""
import pytest

import paper_2407_20496_amd as hinm

P = 0x10000          # never dereferenced
UNSUPPORTED = 5
BIG = 1 << 40


@pytest.mark.parametrize("M,K,N", [(16, 1 << 30, 65), (16, 1 << 29, 200), (1, 1, (1 << 29) - 128), (1, 300, 1 << 27)])
def test_a_layer_refuses_activations_that_quantising_alone_refuses(M, K, N):
    lib = hinm.load_library()
    assert lib.hinm_mx4_quantize(K, N, 1, P, N, hinm.MX4_COLUMNS, P, P, None) == UNSUPPORTED
    assert lib.hinm_mx4_linear(M, K, N, 1, P, P, P, N, P, N, 0, P, BIG, None) == UNSUPPORTED


@pytest.mark.parametrize("K,N", [(1 << 27, 65), (1 << 30, 65), ((1 << 27) + 5, 4096)])
@pytest.mark.parametrize("wanted", ["dw_post", "dgate", "dw_pre"])
def test_gradients_refuse_more_channels_than_one_launch_adds_up(K, N, wanted):
    import ctypes as C
    of = lambda name: P if name == wanted else None
    assert hinm.load_library().hinm_block_norm_grad(K, N, 0, C.c_float(1), P, P, P, P, P, P, P, P, P, P, P, N, P, N, of("dw_post"), of("dgate"),
                                                    None, of("dw_pre"), P, 1 << 50, None) == UNSUPPORTED
