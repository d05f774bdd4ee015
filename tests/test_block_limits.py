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


HELD = [(1, 1), (768, 1), (4096, 1), (4096, 16), (768, 4096), (1024, 100)]
IN_TWO = [(4097, 1), (4097, 16), (4096, 17), (768, 4097), (1025, 17), (16384, 4096)]


def test_a_norm_in_one_launch_asks_for_no_workspace():
    assert [hinm.hinm_block_norm_workspace(*s) for s in HELD] == [0] * len(HELD)
    assert all(hinm.hinm_block_norm_workspace(*s) > 0 for s in IN_TWO)


@pytest.mark.gpu
@pytest.mark.parametrize("K,N", HELD)
def test_a_norm_in_one_launch_takes_no_workspace(K, N):
    import numpy as np
    import torch
    from oracle import block_oracle as orc
    from tests.test_gpu_block_norm import HALF_STEP, SUM
    ld = (N + 7) // 8 * 8
    x, y = (torch.randn(K, ld, device="cuda:0").to(torch.bfloat16) for _ in range(2))
    w = torch.rand(K, device="cuda:0") + 0.5
    h, u = torch.empty_like(x), torch.empty_like(x)
    hinm.hinm_block_norm(K, N, "bf16", 1.0, 1e-5, x, y, w, None, None, w, h, ld, u, ld)
    wide = lambda t: t[:, :N].float().cpu().numpy().astype(np.float64)
    wd = w.cpu().numpy().astype(np.float64)
    want = orc.block_norm(wide(x), wide(y), wd, None, None, wd, 1.0, 1e-5)
    assert (np.abs(wide(h) - want["h"]) <= HALF_STEP["bf16"] * np.abs(want["h"]) + SUM * want["size"]).all()
    of_h = np.sqrt((want["size"] ** 2).mean(axis=0) + 1e-5) * want["rstd_h"]
    assert (np.abs(wide(u) - want["u"]) <= HALF_STEP["bf16"] * np.abs(want["u"])
            + SUM * wd[:, None] * want["rstd_h"] * want["size"] * (1 + of_h)).all()
