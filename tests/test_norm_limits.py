"""Channels' gradients of several strips of tokens are added by workgroups of 1024 threads, 32 channels each, and a launch has less
than 2^32 threads: the same limit for both norms, refused ahead of every launch.  No GPU."""
import ctypes as C

import pytest

import paper_2407_20496_amd as hinm

P = 0x10000  # never dereferenced
UNSUPPORTED, WORKSPACE = 5, 4
MOST = 32 * ((1 << 22) - 1)  # channels; one more needs a workgroup more


def _block_norm_grad(K, N, wanted, ws):
    of = lambda name: P if name == wanted else None
    return hinm.load_library().hinm_block_norm_grad(K, N, 0, C.c_float(1), P, P, P, P, P, P, P, P, P, P, P, N, P, N, of("dw_post"), of("dgate"),
                                                    of("dtoken_gate"), of("dw_pre"), ws, 1 << 60, None)


def _layer_norm_grad(K, N, wanted, ws):
    of = lambda name: P if name == wanted else None
    return hinm.load_library().hinm_layer_norm_grad(K, N, 0, P, N, P, P, P, P, N, P, P, of("dw"), of("db"), ws, 1 << 60, None)


CALLS = [(_block_norm_grad, w) for w in ("dw_post", "dgate", "dw_pre")] + [(_layer_norm_grad, w) for w in ("dw", "db")]


@pytest.mark.parametrize("call,wanted", CALLS)
@pytest.mark.parametrize("N", [65, 4096])
def test_one_workgroup_too_many_is_refused(call, wanted, N):
    assert -(-MOST // 32) * 1024 < 1 << 32 == -(-(MOST + 1) // 32) * 1024
    for K in (MOST + 1, MOST + 31, MOST + 32, 1 << 30):
        assert call(K, N, wanted, P) == UNSUPPORTED, K
    assert call(MOST, N, wanted, None) == WORKSPACE  # the next of the call's checks


@pytest.mark.parametrize("call,wanted", [(_block_norm_grad, "dtoken_gate"), (_block_norm_grad, "nothing"), (_layer_norm_grad, "nothing")])
def test_without_that_launch_there_is_no_such_limit(call, wanted):
    assert call(MOST + 1, 65, wanted, None) == WORKSPACE
    for any_call, w in CALLS:  # one strip has nothing to add
        assert any_call(MOST + 1, 64, w, None) == WORKSPACE
