"""Norms around a block at the ends of their numbers: tokens far larger or smaller than one."""
import numpy as np
import pytest

from oracle import block_oracle as orc
from tests.test_gpu_block_norm import HALF_STEP, SUM, Matrix, _check, _f32, _guarded, _values, _vec, _workspace

pytestmark = pytest.mark.gpu

# root mean squares of tokens: all of bf16's range that leaves their squares, and sums of them over some thousand channels, in float32
SIZES = [1.0, 1e13, 1e14, 1e15, 1e17, 1e-13, 3e-15, 1e5]
# one launch that holds two and four rows a thread, and strips in each layout
SHAPES = [(300, 8, 8), (1500, 8, 8), (1100, 24, 24), (1100, 24, 25), (1100, 72, 128)]


@pytest.mark.parametrize("K,N,ld", SHAPES)
def test_gradients_of_large_and_small_tokens(K, N, ld):
    import paper_2407_20496_amd as hinm
    rng = np.random.default_rng(K + ld)
    size = np.array([SIZES[n % len(SIZES)] for n in range(N)])
    new = lambda s: Matrix(K, N, ld, 0, "bf16", rng.standard_normal((K, N)) * s)
    h, y, du = new(size), new(size[::-1]), new(1.0)
    dx, dy = Matrix(K, N, ld, 0, "bf16"), Matrix(K, N, ld, 0, "bf16")
    rstd = lambda m: (1 / np.sqrt((m.wide ** 2).mean(axis=0))).astype(np.float32)
    ry, rh = rstd(y), rstd(h)
    w_post, w_pre = (1 + 0.3 * rng.standard_normal((2, K))).astype(np.float32)
    gate = rng.random(N).astype(np.float32)
    out = {"dw_post": _guarded(K), "dtoken_gate": _guarded(N), "dw_pre": _guarded(K)}
    hinm.hinm_block_norm_grad(K, N, "bf16", 1.0, h.ptr, y.ptr, _vec(w_post), None, _vec(gate), _vec(w_pre), _vec(ry), _vec(rh), None,
                              du.ptr, dx.ptr, ld, dy.ptr, ld, out["dw_post"], None, out["dtoken_gate"], out["dw_pre"],
                              *_workspace(hinm.hinm_block_norm_grad_workspace(K, N)))
    want = orc.block_norm_grad(h.wide, y.wide, _f32(w_post), None, _f32(gate), _f32(w_pre), _f32(ry), _f32(rh), None, du.wide, 1.0)
    for name, (value, magnitude) in want.items():
        if name in ("dx", "dy"):
            # 2^-134: half a step of the smallest numbers
            got = (dx if name == "dx" else dy).result()
            _check(name, got, value, HALF_STEP["bf16"] * np.abs(value) + SUM * magnitude + 2.0 ** -134)
        else:
            _check(name, _values(out[name], value.size), value, SUM * magnitude)
