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


FAR = [1 << 31, (1 << 32) + 4, (1 << 32) + 64, (1 << 64) + 4, -(1 << 32) + 4, -(1 << 64) + 4]
CALLS = {
    "hinm_mx4_quantize": (lambda r, c: (r, c, "f16", P, BIG, 0, P, P), 2),
    "hinm_mx4_unpack": (lambda r, c: (r, c, "f16", P, P, P, BIG), 2),
    "hinm_mx4_product": (lambda m, n, k: (m, n, k, "f16", P, P, P, P, P, BIG), 3),
    "hinm_mx4_linear": (lambda m, k, n: (m, k, n, "f16", P, P, P, BIG, P, BIG, 0, P, BIG), 3),
    "hinm_block_norm": (lambda k, n: (k, n, "f16", 1.0, 1e-6, P, None, None, None, None, P, P, BIG, P, BIG, None, None, P, BIG), 2),
    "hinm_block_norm_grad": (lambda k, n: (k, n, "f16", 1.0, P, P, None, None, None, P, None, P, P, P, P, BIG, P, BIG, None, None, None, None, P, BIG), 2),
}


@pytest.mark.parametrize("far", FAR)
@pytest.mark.parametrize("which", CALLS)
def test_calls_refuse_sizes_that_32_bits_do_not_hold(which, far):
    """2^32 + 4 rows are not four."""
    arguments, sizes = CALLS[which]
    for i in range(sizes):
        given = [64] * sizes
        given[i] = far
        with pytest.raises(hinm.HinmError) as e:
            getattr(hinm, which)(*arguments(*given), stream=1)
        assert e.value.status == (UNSUPPORTED if far > 0 else 2), i


@pytest.mark.parametrize("far", FAR)
@pytest.mark.parametrize("which,sizes", [("hinm_mx4_sizes", 2), ("hinm_mx4_linear_workspace", 3), ("hinm_block_norm_workspace", 2),
                                         ("hinm_block_norm_grad_workspace", 2)])
def test_questions_refuse_sizes_that_32_bits_do_not_hold(which, sizes, far):
    for i in range(sizes):
        given = [64] * sizes
        given[i] = far
        with pytest.raises(hinm.HinmError) as e:
            getattr(hinm, which)(*given)
        assert e.value.status == (UNSUPPORTED if far > 0 else 2), i


@pytest.mark.parametrize("flags", [1 << 32, (1 << 32) + 1, 1 << 64, -(1 << 32)])
def test_calls_refuse_flags_that_32_bits_do_not_hold(flags):
    for call in (lambda: hinm.hinm_mx4_product(64, 64, 64, "f16", P, P, P, P, P, 64, flags, stream=1),
                 lambda: hinm.hinm_mx4_linear(64, 64, 64, "f16", P, P, P, 64, P, 64, flags, P, BIG, stream=1)):
        with pytest.raises(hinm.HinmError) as e:
            call()
        assert e.value.status == UNSUPPORTED
