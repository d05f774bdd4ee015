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


INF, NAN = float("inf"), float("nan")
# (x in row 7, x in row 200, y in row 7, y in row 200, row 250: gate zero there; token gate); None: as drawn
TOKENS = [(None, None, None, None, None, 1), (INF, None, None, None, None, 1), (-INF, None, None, None, None, -0.5), (INF, None, 0, None, None, 1),
          (INF, -INF, None, None, None, 1), (None, None, INF, None, None, 1), (INF, None, -INF, None, None, 1), (INF, None, INF, None, None, 1),
          (INF, None, None, -INF, None, 1), (NAN, None, None, None, None, 1), (None, None, None, NAN, None, 1), (None, None, INF, None, None, 0),
          (INF, None, INF, None, None, -1), (INF, None, -INF, None, None, -1), (None, None, None, None, ("y", INF), 1),
          (None, None, None, None, ("x", -INF), 1), (INF, INF, -INF, INF, None, 1), (-INF, INF, INF, -INF, None, -2), (INF, None, 0, None, None, 0)]


def _same(name, got, want, bound):
    """Infinities and NaN in the same places, everything else within the bound; exact where the magnitudes are infinite."""
    bound = np.where(np.isfinite(bound), bound, 0)
    assert np.array_equal(np.isnan(got), np.isnan(want)), (name, np.argwhere(np.isnan(got) != np.isnan(want))[:4])
    plain = np.isfinite(want)
    assert np.array_equal(got[np.isinf(want)], want[np.isinf(want)]) and (np.abs(got - want)[plain] <= bound[plain]).all(), name


@pytest.mark.parametrize("scale", [1.0, -0.75, 0.0])
@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("K,ld,in_place", [(300, 24, False), (1100, 24, False), (1100, 19, False), (1100, 64, False), (1100, 64, True), (9000, 24, True),
                                           (9000, 1, False)])
def test_infinities_are_those_of_the_formula(K, ld, in_place, post, scale):
    """One launch that holds the tokens, two in every layout, and tokens one by one (ld = 1) agree on what an infinity does."""
    import paper_2407_20496_amd as hinm
    rng = np.random.default_rng(K)
    N = len(TOKENS)
    x, y = rng.standard_normal((2, K, N))
    for n, (x7, x200, y7, y200, at_zero, _) in enumerate(TOKENS):
        for a, row, v in ((x, 7, x7), (x, 200, x200), (y, 7, y7), (y, 200, y200)):
            if v is not None:
                a[row, n] = v
        if at_zero:
            (x if at_zero[0] == "x" else y)[250, n] = at_zero[1]
    token_gate = np.array([t[5] for t in TOKENS], dtype=np.float32)
    gate, w = rng.standard_normal(K).astype(np.float32), (1 + 0.3 * rng.standard_normal(K)).astype(np.float32)
    gate[7], gate[200], gate[250] = 1.5, 0.5, 0
    w_post = w[::-1].copy() if post else None
    eps = np.float32(1e-5)
    for cols in ([slice(n, n + 1) for n in range(N)] if ld == 1 else [slice(0, N)]):
        n = x[:, cols].shape[1]
        X, Y = Matrix(K, n, ld, 0, "bf16", x[:, cols]), Matrix(K, n, ld, 0, "bf16", y[:, cols])
        h, u = (X, Y) if in_place else (Matrix(K, n, ld, 0, "bf16"), Matrix(K, n, ld, 0, "bf16"))
        ry, rh = _guarded(n, post), _guarded(n)
        hinm.hinm_block_norm(K, n, "bf16", scale, float(eps), X.ptr, Y.ptr, _vec(w_post), _vec(gate), _vec(token_gate[cols]), _vec(w), h.ptr, ld,
                             u.ptr, ld, ry, rh, *_workspace(hinm.hinm_block_norm_workspace(K, n)))
        with np.errstate(all="ignore"):
            want = orc.block_norm(X.wide, Y.wide, _f32(w_post), _f32(gate), _f32(token_gate[cols]), _f32(w), scale, float(eps))
            of_h = np.sqrt((want["size"] ** 2).mean(axis=0) + eps) * want["rstd_h"]
            background = 0x7FFF if in_place else 0x1234
            _same("h", h.result(background), want["h"], HALF_STEP["bf16"] * np.abs(want["h"]) + SUM * want["size"])
            _same("rstd_h", _values(rh, n), want["rstd_h"], SUM * of_h * want["rstd_h"])
            _same("u", u.result(background), want["u"],
                  HALF_STEP["bf16"] * np.abs(want["u"]) + SUM * np.abs(w)[:, None] * want["rstd_h"] * want["size"] * (1 + of_h))
            if post:
                _same("rstd_y", _values(ry, n), want["rstd_y"], SUM * want["rstd_y"])


@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("K,N,ld", [(300, 9, 16), (3000, 9, 16), (1100, 27, 32), (1100, 27, 27), (1100, 81, 128), (5000, 1, 1)])
def test_large_and_small_tokens(K, N, ld, post):
    """Down to 1e-17 without eps, up to 1e17, in every kernel."""
    import paper_2407_20496_amd as hinm
    rng = np.random.default_rng(K + N)
    sizes = [1e17, 1e-17, 1e15, 1e-13, 1.0, 1e13, 1e5, 1e-5, 3e-15]
    for first in range(len(sizes) if N == 1 else 1):
        size = np.array([sizes[(first + n) % len(sizes)] for n in range(N)])
        x, y = (Matrix(K, N, ld, 0, "bf16", rng.standard_normal((K, N)) * size) for _ in range(2))
        h, u = Matrix(K, N, ld, 0, "bf16"), Matrix(K, N, ld, 0, "bf16")
        w_post, w_pre = (1 + 0.3 * rng.standard_normal((2, K))).astype(np.float32)
        ry, rh = _guarded(N, post), _guarded(N)
        given = w_post if post else None
        hinm.hinm_block_norm(K, N, "bf16", 0.75, 0.0, x.ptr, y.ptr, _vec(given), None, None, _vec(w_pre), h.ptr, ld, u.ptr, ld, ry, rh,
                             *_workspace(hinm.hinm_block_norm_workspace(K, N)))
        want = orc.block_norm(x.wide, y.wide, _f32(given), None, None, _f32(w_pre), 0.75, 0.0)
        of_h = np.sqrt((want["size"] ** 2).mean(axis=0)) * want["rstd_h"]
        _check("h", h.result(), want["h"], HALF_STEP["bf16"] * np.abs(want["h"]) + SUM * want["size"])
        _check("rstd_h", _values(rh, N), want["rstd_h"], SUM * of_h * want["rstd_h"])
        _check("u", u.result(), want["u"], HALF_STEP["bf16"] * np.abs(want["u"])
               + SUM * np.abs(_f32(w_pre))[:, None] * want["rstd_h"] * want["size"] * (1 + of_h))
        if post:
            _check("rstd_y", _values(ry, N), want["rstd_y"], SUM * want["rstd_y"])
