"""Host-side checks of the dense layers' and layer norm's entry points: sizes, refusals, and which forms of the products the GPU
tests reach.  No GPU: every call is refused before anything is launched."""
import ctypes as C

import pytest

import paper_2407_20496_amd as hinm

P = 0x10000          # never dereferenced
OK, NULL, SHAPE, DTYPE, WORKSPACE, UNSUPPORTED = 0, 1, 2, 3, 4, 5
BIG = 1 << 40
FAR = 1 << 33


def _refused(call, good, **changes):
    args = dict(good)
    args.update(changes)
    return call(*args.values(), None)


@pytest.mark.parametrize("change,status", [
    ({"dtype": 7}, DTYPE), ({"M": 0}, SHAPE), ({"K": -1}, SHAPE), ({"N": 0}, SHAPE), ({"W": None}, NULL), ({"X": None}, NULL), ({"Y": None}, NULL),
    ({"ldw": 63}, SHAPE), ({"ldx": 7}, SHAPE), ({"ldy": 7}, SHAPE), ({"ldr": 7}, SHAPE), ({"W": P + 1}, SHAPE), ({"X": P + 1}, SHAPE),
    ({"R": P + 1}, SHAPE), ({"Z": P + 1}, SHAPE), ({"Y": P + 1}, SHAPE), ({"bias": P + 2}, SHAPE), ({"flags": 2, "Y": P + 2}, SHAPE),
    ({"flags": 1 | 4}, UNSUPPORTED), ({"flags": 8 | 16}, UNSUPPORTED), ({"flags": 32}, UNSUPPORTED), ({"flags": 0x100}, UNSUPPORTED),
    ({"M": (1 << 30) + 1}, UNSUPPORTED), ({"K": (1 << 30) + 1, "ldw": FAR}, UNSUPPORTED), ({"N": (1 << 30) + 1, "ldx": FAR, "ldy": FAR, "ldr": FAR}, UNSUPPORTED),
    ({"M": 1 << 18, "N": 1 << 18, "ldx": FAR, "ldy": FAR, "ldr": FAR}, UNSUPPORTED)])
def test_linear_refusals(change, status):
    good = dict(M=16, K=64, N=8, dtype=1, W=P, ldw=64, X=P, ldx=8, bias=P, R=P, ldr=8, Z=P, Y=P, ldy=8, flags=4, ws=P, bytes=BIG)
    assert _refused(hinm.load_library().hinm_linear, good, **change) == status


@pytest.mark.parametrize("change,status", [
    ({"dtype": -1}, DTYPE), ({"M": 0}, SHAPE), ({"K": 0}, SHAPE), ({"N": -5}, SHAPE), ({"W": None}, NULL), ({"X": None}, NULL), ({"Z": None}, NULL),
    ({"dY": None}, NULL), ({"dX": None, "dW": None, "db": None}, NULL), ({"ldw": 63}, SHAPE), ({"ldx": 7}, SHAPE), ({"ldy": 7}, SHAPE),
    ({"W": P + 1}, SHAPE), ({"X": P + 1}, SHAPE), ({"Z": P + 1}, SHAPE), ({"dY": P + 1}, SHAPE), ({"dX": P + 1}, SHAPE), ({"dW": P + 1}, SHAPE),
    ({"db": P + 2}, SHAPE), ({"flags": 2, "dW": P + 2}, SHAPE), ({"flags": 5}, UNSUPPORTED), ({"flags": 64}, UNSUPPORTED),
    ({"M": (1 << 30) + 1}, UNSUPPORTED), ({"M": 1 << 18, "K": 1 << 18, "ldw": FAR}, UNSUPPORTED), ({"ws": None}, WORKSPACE), ({"ws": P + 128}, WORKSPACE), ({"bytes": 255}, WORKSPACE)])
def test_linear_grad_refusals(change, status):
    good = dict(M=16, K=64, N=8, dtype=1, W=P, ldw=64, X=P, ldx=8, Z=P, dY=P, ldy=8, dX=P, dW=P, db=P, flags=4, ws=P, bytes=BIG)
    assert _refused(hinm.load_library().hinm_linear_grad, good, **change) == status


@pytest.mark.parametrize("change,status", [
    ({"dtype": 7}, DTYPE), ({"K": 0}, SHAPE), ({"N": 0}, SHAPE), ({"x": None}, NULL), ({"u": None}, NULL), ({"ldx": 7}, SHAPE), ({"ldu": 7}, SHAPE),
    ({"x": P + 1}, SHAPE), ({"u": P + 1}, SHAPE), ({"w": P + 2}, SHAPE), ({"b": P + 2}, SHAPE), ({"mean": P + 2}, SHAPE), ({"rstd": P + 2}, SHAPE),
    ({"N": (1 << 22) + 1, "ldx": FAR, "ldu": FAR}, UNSUPPORTED), ({"K": (1 << 30) + 1}, UNSUPPORTED)])
def test_layer_norm_refusals(change, status):
    good = dict(K=64, N=8, dtype=0, eps=C.c_float(0), x=P, ldx=8, w=P, b=P, u=P, ldu=8, mean=P, rstd=P, ws=P, bytes=BIG)
    assert _refused(hinm.load_library().hinm_layer_norm, good, **change) == status


@pytest.mark.parametrize("change,status", [
    ({"dtype": 7}, DTYPE), ({"K": 0}, SHAPE), ({"N": 0}, SHAPE), ({"x": None}, NULL), ({"mean": None}, NULL), ({"rstd": None}, NULL),
    ({"du": None}, NULL), ({"dx": None, "dw": None, "db": None}, NULL), ({"ldx": 7}, SHAPE), ({"ldu": 7}, SHAPE), ({"x": P + 1}, SHAPE),
    ({"du": P + 1}, SHAPE), ({"dh": P + 1}, SHAPE), ({"dx": P + 1}, SHAPE), ({"w": P + 2}, SHAPE), ({"mean": P + 1}, SHAPE), ({"rstd": P + 2}, SHAPE),
    ({"dw": P + 2}, SHAPE), ({"db": P + 2}, SHAPE), ({"N": (1 << 22) + 1, "ldx": FAR, "ldu": FAR}, UNSUPPORTED),
    ({"K": 1 << 27, "N": 65, "ldx": 72, "ldu": 72}, UNSUPPORTED)])
def test_layer_norm_grad_refusals(change, status):
    good = dict(K=64, N=8, dtype=0, x=P, ldx=8, w=P, mean=P, rstd=P, du=P, ldu=8, dh=P, dx=P, dw=P, db=P, ws=P, bytes=BIG)
    assert _refused(hinm.load_library().hinm_layer_norm_grad, good, **change) == status


def test_workspaces():
    lib, n = hinm.load_library(), C.c_size_t(0)
    for size in (lib.hinm_linear_workspace, lib.hinm_linear_grad_workspace):
        assert size(1, 1, 1, None) == NULL
        assert size(0, 1, 1, C.byref(n)) == SHAPE
        assert size(1, (1 << 30) + 1, 1, C.byref(n)) == UNSUPPORTED
    assert lib.hinm_linear_workspace(1 << 18, 64, 1 << 18, C.byref(n)) == UNSUPPORTED
    assert lib.hinm_linear_grad_workspace(1 << 18, 1 << 18, 64, C.byref(n)) == UNSUPPORTED
    for size in (lib.hinm_layer_norm_workspace, lib.hinm_layer_norm_grad_workspace):
        assert size(1, 1, None) == NULL
        assert size(1, 0, C.byref(n)) == SHAPE
        assert size(1, (1 << 22) + 1, C.byref(n)) == UNSUPPORTED
    f = C.c_float(1)
    for need, call in ((hinm.hinm_linear_workspace(256, 4096, 64),
                        lambda ws, b: lib.hinm_linear(256, 4096, 64, 0, P, 4096, P, 64, None, None, 0, None, P, 64, 0, ws, b, None)),
                       (hinm.hinm_linear_grad_workspace(256, 4096, 64),
                        lambda ws, b: lib.hinm_linear_grad(256, 4096, 64, 0, P, 4096, P, 64, P, P, 64, P, P, P, 1, ws, b, None)),
                       (hinm.hinm_layer_norm_workspace(4096, 100),
                        lambda ws, b: lib.hinm_layer_norm(4096, 100, 0, f, P, 104, P, P, P, 104, P, P, ws, b, None)),
                       (hinm.hinm_layer_norm_grad_workspace(4096, 100),
                        lambda ws, b: lib.hinm_layer_norm_grad(4096, 100, 0, P, 104, P, P, P, P, 104, P, P, P, P, ws, b, None))):
        assert need > 0
        assert call(None, need) == WORKSPACE
        assert call(P, need - 1) == WORKSPACE
        assert call(P + 128, need) == WORKSPACE


def test_python_calls_raise_with_the_status():
    for call in (lambda: hinm.hinm_linear(16, 64, 8, "bf16", P, 64, P, 8, None, None, 0, None, None, 8, stream=1),
                 lambda: hinm.hinm_linear_grad(16, 64, 8, "bf16", P, 64, P, 8, None, None, 8, P, P, stream=1),
                 lambda: hinm.hinm_layer_norm(64, 8, "bf16", 1e-5, None, 8, None, None, P, 8, stream=1),
                 lambda: hinm.hinm_layer_norm_grad(64, 8, "bf16", P, 8, None, P, P, None, 8, None, P, stream=1)):
        with pytest.raises(hinm.HinmError) as e:
            call()
        assert e.value.status == NULL
    with pytest.raises(ValueError):
        hinm.hinm_linear(16, 64, 8, "f32", P, 64, P, 8, None, None, 0, None, P, 8, stream=1)
    with pytest.raises(TypeError):
        hinm.hinm_layer_norm(64, 8, "bf16", "small", P, 8, None, None, P, 8, stream=1)
    # sizes that 32 bits do not hold are refused, and not taken as what is left of them
    with pytest.raises(hinm.HinmError) as e:
        hinm.hinm_linear((1 << 32) + 16, 64, 8, "bf16", P, 64, P, 8, None, None, 0, None, P, 8, stream=1)
    assert e.value.status == UNSUPPORTED


def test_a_launch_has_less_than_32_bits_of_threads():
    """Few tokens have 16 rows a workgroup, of up to 1024 threads; channels' gradients 32 channels a workgroup of as many."""
    lib, n = hinm.load_library(), C.c_size_t(0)
    most = 16 * ((1 << 22) - 8) - 1
    assert -(-most // 16) * 1024 < 1 << 32
    for tokens in (1, 16):
        assert lib.hinm_linear_workspace(most, 1, tokens, C.byref(n)) == OK
        for M in (most + 1, 1 << 26, (1 << 28) - 64):
            assert lib.hinm_linear_workspace(M, 1, tokens, C.byref(n)) == UNSUPPORTED
            assert lib.hinm_linear(M, 1, tokens, 1, P, 8, P, 16, None, None, 0, None, P, 16, 0, P, BIG, None) == UNSUPPORTED
    assert lib.hinm_linear_workspace(1 << 26, 1, 17, C.byref(n)) == OK
    K = (1 << 27) - 31
    assert lib.hinm_layer_norm_grad(K, 65, 0, P, 72, P, P, P, P, 72, P, P, P, P, P, 1 << 60, None) == UNSUPPORTED
