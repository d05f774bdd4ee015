"""What hinm_calib_linear_plan says of a layer's gradients is what the call launches: dZ always lies in whole pieces, X of 33 to 64
tokens is copied to whole pieces where it does not.  No GPU."""
import re

import pytest

import paper_2407_20496_amd as hinm

IN, WEIGHTS, BOTH = 1, 2, 3
launches = lambda M, K, N, which, aligned, dtype="f16": [l for l in re.split(r"[;\n]\s*", hinm.hinm_calib_linear_plan(M, K, N, dtype, which, aligned)) if l]
name = lambda l: l.split("<")[0].split(" ")[0]


@pytest.mark.parametrize("M,K,N", [(256, 256, 40), (1000, 520, 33), (4096, 4096, 64), (7, 65, 50)])
def test_activations_of_few_tokens_are_copied(M, K, N):
    got = launches(M, K, N, WEIGHTS, False)
    assert name(got[0]) == "linear_copy_kernel" and "GUARDED=0" in got[1]
    assert got[1:] == launches(M, K, N, WEIGHTS, True)


@pytest.mark.parametrize("M,K,N", [(256, 256, 65), (768, 771, 4096), (4096, 4096, 1000)])
def test_activations_of_many_tokens_are_taken_as_they_lie(M, K, N):
    got = launches(M, K, N, WEIGHTS, False)
    assert name(got[0]) == "linear_tile_kernel" and "GUARDED=1" in got[0]


@pytest.mark.parametrize("M,K,N", [(768, 771, 4096), (4097, 4097, 600), (4096, 4096, 2048), (100, 99, 20), (256, 256, 40), (5, 33, 300)])
def test_weights_apart_are_of_no_account_to_their_gradient(M, K, N):
    """With both gradients W alone is unaligned, which the product of dZ and X does not read."""
    of_x, of_w, both = launches(M, K, N, IN, False), launches(M, K, N, WEIGHTS, True), launches(M, K, N, BOTH, False)
    assert both == of_x + of_w
    assert "GUARDED=1" not in "".join(of_w)


@pytest.mark.parametrize("M,K,N", [(768, 768, 4096), (64, 64, 9)])
def test_one_launch_for_both(M, K, N):
    assert [name(l) for l in launches(M, K, N, BOTH, True)] == ["linear_pair_kernel"]
    assert "linear_pair_kernel" not in [name(l) for l in launches(M, K, N, BOTH, False)]
