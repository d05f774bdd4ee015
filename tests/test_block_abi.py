"""Host-side checks of the entry points of the 4-bit form and of a block's norms: sizes and refusals.  No GPU: every case
is refused before anything is launched."""
import ctypes as C

import pytest

import paper_2407_20496_amd as hinm
from paper_2407_20496_amd import binding  # noqa: F401

P = 0x10000          # never dereferenced
OK, NULL, SHAPE, DTYPE, WORKSPACE, UNSUPPORTED = 0, 1, 2, 3, 4, 5
BIG = 1 << 40


@pytest.mark.parametrize("rows,length,want", [(1, 1, (4096, 512)), (32, 256, (4096, 512)), (33, 257, (16384, 1024)),
                                              (64, 512, (16384, 1024)), (2, 513, (12288, 1024)),
                                              (11008, 4096, (11008 * 2048, 11008 * 128)),
                                              (1 << 20, 1 << 20, (1 << 39, 1 << 35))])
def test_sizes(rows, length, want):
    assert hinm.hinm_mx4_sizes(rows, length) == want


def test_bad_sizes():
    for rows, length in ((0, 1), (1, 0), (-1, 5), (5, -1)):
        with pytest.raises(hinm.HinmError) as e:
            hinm.hinm_mx4_sizes(rows, length)
        assert e.value.status == SHAPE
    lib = hinm.load_library()
    assert lib.hinm_mx4_sizes(4, 4, None, None) == OK
    assert lib.hinm_mx4_linear_workspace(1, 1, 1, None) == NULL
    assert lib.hinm_block_norm_workspace(1, 1, None) == NULL
    assert lib.hinm_block_norm_grad_workspace(1, 1, None) == NULL
    n = C.c_size_t(0)
    assert lib.hinm_mx4_linear_workspace(0, 1, 1, C.byref(n)) == SHAPE
    assert lib.hinm_block_norm_workspace(0, 1, C.byref(n)) == SHAPE
    assert lib.hinm_block_norm_grad_workspace(1, -1, C.byref(n)) == SHAPE
    assert lib.hinm_block_norm_workspace(1, (1 << 22) + 1, C.byref(n)) == UNSUPPORTED
    assert lib.hinm_block_norm_grad_workspace((1 << 30) + 1, 1, C.byref(n)) == UNSUPPORTED
    assert lib.hinm_mx4_linear_workspace(1, (1 << 30) + 1, 1, C.byref(n)) == UNSUPPORTED


def _refused(call, good, **changes):
    args = dict(good)
    args.update(changes)
    return call(*args.values(), None)


@pytest.mark.parametrize("change,status", [
    ({"dtype": 2}, DTYPE), ({"rows": 0}, SHAPE), ({"cols": -1}, SHAPE), ({"src": None}, NULL), ({"codes": None}, NULL),
    ({"scales": None}, NULL), ({"ld": 63}, SHAPE), ({"src": P + 1}, SHAPE), ({"codes": P + 8}, SHAPE), ({"scales": P + 4}, SHAPE),
    ({"along": 2}, UNSUPPORTED), ({"along": -1}, UNSUPPORTED), ({"rows": (1 << 30) + 1}, UNSUPPORTED), ({"rows": 1 << 30}, UNSUPPORTED),
    ({"rows": 1 << 30, "cols": 1, "ld": 2, "along": 1}, UNSUPPORTED), ({"rows": 1, "cols": (1 << 30) + 1, "ld": BIG}, UNSUPPORTED)])
def test_quantize_refusals(change, status):
    good = dict(rows=32, cols=64, dtype=0, src=P, ld=64, along=0, codes=P, scales=P)
    assert _refused(hinm.load_library().hinm_mx4_quantize, good, **change) == status


@pytest.mark.parametrize("change,status", [
    ({"dtype": -1}, DTYPE), ({"rows": 0}, SHAPE), ({"length": 0}, SHAPE), ({"dst": None}, NULL), ({"codes": None}, NULL),
    ({"ld": 63}, SHAPE), ({"dst": P + 1}, SHAPE), ({"codes": P + 1}, SHAPE), ({"rows": 1 << 30}, UNSUPPORTED),
    ({"length": (1 << 30) + 1, "ld": BIG}, UNSUPPORTED)])
def test_unpack_refusals(change, status):
    good = dict(rows=32, length=64, dtype=0, codes=P, scales=P, dst=P, ld=64)
    assert _refused(hinm.load_library().hinm_mx4_unpack, good, **change) == status


@pytest.mark.parametrize("change,status", [
    ({"dtype": 7}, DTYPE), ({"M": 0}, SHAPE), ({"N": 0}, SHAPE), ({"K": -4}, SHAPE), ({"ac": None}, NULL), ({"asc": None}, NULL),
    ({"bc": None}, NULL), ({"bs": None}, NULL), ({"Y": None}, NULL), ({"ldy": 7}, SHAPE), ({"bc": P + 8}, SHAPE), ({"Y": P + 1}, SHAPE),
    ({"flags": 4}, UNSUPPORTED), ({"flags": 0x100}, UNSUPPORTED), ({"flags": 2, "Y": P + 2}, SHAPE),
    ({"M": (1 << 31) - 1, "N": (1 << 31) - 1, "ldy": BIG}, UNSUPPORTED), ({"M": 1 << 30, "N": 1, "ldy": 1}, UNSUPPORTED),
    ({"K": (1 << 30) + 1}, UNSUPPORTED), ({"M": 1 << 20, "N": 1 << 20, "ldy": BIG}, UNSUPPORTED)])
def test_product_refusals(change, status):
    good = dict(M=16, N=8, K=64, dtype=1, ac=P, asc=P, bc=P, bs=P, Y=P, ldy=8, flags=0)
    assert _refused(hinm.load_library().hinm_mx4_product, good, **change) == status


@pytest.mark.parametrize("change,status", [
    ({"dtype": 7}, DTYPE), ({"M": 0}, SHAPE), ({"X": None}, NULL), ({"codes": None}, NULL), ({"ldx": 7}, SHAPE), ({"ldy": 7}, SHAPE),
    ({"X": P + 1}, SHAPE), ({"flags": 8}, UNSUPPORTED), ({"ws": None}, WORKSPACE), ({"ws": P + 128}, WORKSPACE),
    ({"bytes": 4096 + 511}, WORKSPACE)])
def test_linear_refusals(change, status):
    good = dict(M=16, K=64, N=8, dtype=1, codes=P, scales=P, X=P, ldx=8, Y=P, ldy=8, flags=0, ws=P, bytes=BIG)
    assert _refused(hinm.load_library().hinm_mx4_linear, good, **change) == status


@pytest.mark.parametrize("change,status", [
    ({"dtype": 7}, DTYPE), ({"K": 0}, SHAPE), ({"N": 0}, SHAPE), ({"N": (1 << 22) + 1, "ls": BIG, "lb": BIG}, UNSUPPORTED),
    ({"x": None}, NULL), ({"y": None}, NULL), ({"y": None, "w_post": None}, NULL), ({"y": None, "w_post": None, "gate": None}, NULL),
    ({"u": None}, NULL), ({"w_pre": None, "h": None}, NULL), ({"ls": 7}, SHAPE), ({"lb": 7}, SHAPE), ({"x": P + 1}, SHAPE),
    ({"u": P + 1}, SHAPE), ({"gate": P + 2}, SHAPE), ({"ry": P + 2}, SHAPE)])
def test_block_norm_refusals(change, status):
    good = dict(K=64, N=8, dtype=0, scale=C.c_float(1), eps=C.c_float(0), x=P, y=P, w_post=P, gate=P, token_gate=P, w_pre=P, h=P,
                ls=8, u=P, lb=8, ry=P, rh=P, ws=P, bytes=BIG)
    assert _refused(hinm.load_library().hinm_block_norm, good, **change) == status


@pytest.mark.parametrize("change,status", [
    ({"dtype": 7}, DTYPE), ({"K": 0}, SHAPE), ({"N": 0}, SHAPE), ({"h": None}, NULL), ({"du": None}, NULL), ({"rh": None}, NULL),
    ({"w_pre": None}, NULL), ({"w_pre": None, "du": None, "dh": None}, NULL), ({"y": None}, NULL), ({"ry": None}, NULL),
    ({"w_post": None}, NULL), ({"gate": None}, NULL), ({"token_gate": None}, NULL), ({"ls": 7}, SHAPE), ({"lb": 7}, SHAPE),
    ({"dh": P + 1}, SHAPE), ({"dy": P + 1}, SHAPE), ({"dgate": P + 2}, SHAPE)])
def test_block_norm_grad_refusals(change, status):
    good = dict(K=64, N=8, dtype=0, scale=C.c_float(1), h=P, y=P, w_post=P, gate=P, token_gate=P, w_pre=P, ry=P, rh=P, dh=P, du=P,
                dx=P, ls=8, dy=P, lb=8, dw_post=P, dgate=P, dtoken=P, dw_pre=P, ws=P, bytes=BIG)
    assert _refused(hinm.load_library().hinm_block_norm_grad, good, **change) == status


def test_workspaces_are_asked_for():
    lib = hinm.load_library()
    need = hinm.hinm_block_norm_grad_workspace(4096, 100)
    assert need > 0
    f = C.c_float(1)
    call = lambda ws, n: lib.hinm_block_norm_grad(4096, 100, 0, f, P, P, P, P, P, P, P, P, P, P, P, 104, P, 104, P, P, P, P, ws, n, None)
    assert call(None, need) == WORKSPACE
    assert call(P, need - 1) == WORKSPACE
    assert call(P + 128, need) == WORKSPACE
    need = hinm.hinm_block_norm_workspace(16384, 4096)
    call = lambda ws, n: lib.hinm_block_norm(16384, 4096, 0, f, f, P, P, P, P, P, P, P, 4096, P, 4096, P, P, ws, n, None)
    if need:
        assert call(None, need) == WORKSPACE
        assert call(P, need - 1) == WORKSPACE
        assert call(P + 128, need) == WORKSPACE


def test_python_calls_raise_with_the_status():
    with pytest.raises(hinm.HinmError) as e:
        hinm.hinm_mx4_quantize(4, 64, "f16", P, 64, 7, P, P, stream=1)
    assert e.value.status == UNSUPPORTED and "hinm_mx4_quantize" in str(e.value)
    with pytest.raises(ValueError):
        hinm.hinm_mx4_unpack(4, 64, "f32", P, P, P, 64, stream=1)
    with pytest.raises(hinm.HinmError):
        hinm.hinm_mx4_linear(16, 64, 8, "bf16", P, P, P, 8, P, 8, 0, None, 0, stream=1)
    with pytest.raises(hinm.HinmError):
        hinm.hinm_block_norm(64, 8, "bf16", 1.0, 1e-6, None, None, None, None, None, None, P, 8, None, 8, stream=1)
    with pytest.raises(hinm.HinmError):
        hinm.hinm_block_norm_grad(64, 8, "bf16", 1.0, None, None, None, None, None, None, None, None, None, None, None, 8, None, 8,
                                  stream=1)
    with pytest.raises(TypeError):
        hinm.hinm_block_norm(64, 8, "bf16", "one", 1e-6, P, P, None, None, None, None, P, 8, None, 8, stream=1)
