"""CPU oracle of the operators around the compressed layers: microscaled 4-bit form, its product, norms around a block.

Plain numpy in binary64, written from the formulas in include/hinm.h; test infrastructure only.  Beside a value the
oracle gives, where a kernel sums in fp32, the sum of the magnitudes that meet in it: rounding errors are bounded by a
number of roundings times that.
"""
from __future__ import annotations

import numpy as np

LEVELS = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=np.float64)
VALUES = np.concatenate([LEVELS, -LEVELS])


def code_pitch(length: int) -> int:
    """Bytes of a row's codes: whole lines of 256 values."""
    return (length + 255) // 256 * 128


def scale_pitch(length: int) -> int:
    return (length + 511) // 512 * 16


def to_memory(codes: np.ndarray, scales: np.ndarray, fill: int = 0):
    """A form with its rows one after the other, as everywhere in this module -> as it lies in memory; rows that only fill
    the last block of 32 hold `fill` in every byte."""
    rows = codes.shape[0]
    rb = (rows + 31) // 32
    grow = lambda a: np.concatenate([a, np.full((32 * rb - rows, a.shape[1]), fill, dtype=np.uint8)])
    c = grow(codes).reshape(rb, 32, -1, 2, 2, 2, 16)     # rows, line, then the bits of p (4: a, 2: b, 1: c), 16 bytes
    c = c.transpose(2, 0, 3, 5, 4, 1, 6)                 # [line][rb][a][c][b][row][16]
    s = grow(scales).reshape(rb, 32, -1, 16).transpose(2, 0, 1, 3)
    return np.ascontiguousarray(c).reshape(-1), np.ascontiguousarray(s).reshape(-1)


def from_memory(codes: np.ndarray, scales: np.ndarray, rows: int):
    rb = (rows + 31) // 32
    c = codes.reshape(-1, rb, 2, 2, 2, 32, 16).transpose(1, 5, 0, 2, 4, 3, 6)
    s = scales.reshape(-1, rb, 32, 16).transpose(1, 2, 0, 3)
    return np.ascontiguousarray(c).reshape(32 * rb, -1), np.ascontiguousarray(s).reshape(32 * rb, -1)


def scale_place(block: int) -> int:
    return block // 16 * 16 + 4 * (block % 4) + block % 16 // 4


def quantize_rows(X: np.ndarray):
    """float64 [rows][length] (what the 16-bit values stand for) -> (codes uint8 [rows][code_pitch], scales uint8
    [rows][scale_pitch]), one value after the other."""
    rows, length = X.shape
    codes = np.zeros((rows, code_pitch(length)), dtype=np.uint8)
    scales = np.full((rows, scale_pitch(length)), 127, dtype=np.uint8)
    middles = (LEVELS[:-1] + LEVELS[1:]) / 2
    for j in range((length + 31) // 32):
        B = X[:, 32 * j:32 * j + 32]
        with np.errstate(invalid="ignore"):
            most = np.abs(B).max(axis=1)
        bad = ~np.isfinite(B).all(axis=1)
        exponent = np.frexp(np.where(bad, 1.0, most))[1] - 1              # floor(log2) of the largest magnitude
        e = np.where(most == 0, 0, np.maximum(exponent - 2 + 127, 0))
        e = np.where(bad, 255, e)
        scales[:, scale_place(j)] = e
        A = np.where(bad[:, None], 0.0, np.abs(B)) / 2.0 ** (np.minimum(e, 254) - 127.0)[:, None]
        place = (A[:, :, None] > middles).sum(axis=2)
        tie = (A[:, :, None] == middles).any(axis=2)
        place = np.where(tie & (place % 2 == 1), place + 1, place)        # the lower neighbour is the odd one: go up
        c = np.where(bad[:, None], 0, place | np.where(np.signbit(B), 8, 0)).astype(np.uint8)
        for i in range(c.shape[1]):
            codes[:, (32 * j + i) // 2] |= c[:, i] << (4 * (i % 2))
    return codes, scales


def values(codes: np.ndarray, scales: np.ndarray, length: int) -> np.ndarray:
    """What a 4-bit form stands for, float64 [rows][length]."""
    nibbles = np.empty((codes.shape[0], codes.shape[1] * 2), dtype=np.uint8)
    nibbles[:, 0::2] = codes & 15
    nibbles[:, 1::2] = codes >> 4
    k = np.arange(length)
    block = k // 32
    e = scales[:, block // 16 * 16 + 4 * (block % 4) + block % 16 // 4].astype(np.float64)
    return np.where(e == 255, np.nan, VALUES[nibbles[:, :length]] * 2.0 ** (e - 127))


def product(A: np.ndarray, B: np.ndarray, relu: bool = False):
    """(A B^T, sum of magnitudes)."""
    Y = A @ B.T
    with np.errstate(invalid="ignore"):
        return (np.where(Y < 0, 0.0, Y) if relu else Y), np.abs(A) @ np.abs(B).T


def _col(v, K):
    return np.ones((K, 1)) if v is None else np.asarray(v, dtype=np.float64).reshape(K, 1)


def _row(v, N):
    return np.ones((1, N)) if v is None else np.asarray(v, dtype=np.float64).reshape(1, N)


def block_norm(x, y, w_post, gate, token_gate, w_pre, scale, eps):
    """{h, u, rstd_y, rstd_h} and the magnitudes of h's two summands, float64 [K][N] inputs."""
    K, N = x.shape
    h, size = scale * x, np.abs(scale * x)
    rstd_y = rstd_h = u = None
    if y is not None:
        if w_post is not None:
            rstd_y = 1 / np.sqrt((y * y).mean(axis=0) + eps)
        branch = _col(gate, K) * _col(w_post, K) * _row(token_gate, N) * _row(rstd_y, N) * y
        h, size = h + branch, size + np.abs(branch)
    if w_pre is not None:
        rstd_h = 1 / np.sqrt((h * h).mean(axis=0) + eps)
        u = _col(w_pre, K) * _row(rstd_h, N) * h
    return {"h": h, "u": u, "rstd_y": rstd_y, "rstd_h": rstd_h, "size": size}


def block_norm_grad(h, y, w_post, gate, token_gate, w_pre, rstd_y, rstd_h, dh, du, scale):
    """Gradients by the formulas, each with the sum of magnitudes: {name: (value, magnitude)}."""
    given = next(t for t in (dh, du) if t is not None)
    K, N = given.shape
    d = np.zeros((K, N)) if dh is None else dh
    size = np.abs(d)
    out = {}
    w, wp, g, t = _col(w_pre, K), _col(w_post, K), _col(gate, K), _row(token_gate, N)
    rh, ry = _row(rstd_h, N), _row(rstd_y, N)
    if w_pre is not None:
        out["dw_pre"] = ((du * h * rh).sum(axis=1), np.abs(du * h * rh).sum(axis=1))
        s1, m1 = (w * du * h).sum(axis=0), np.abs(w * du * h).sum(axis=0)
        d = d + rh * w * du - h * rh ** 3 * s1 / K
        size = size + np.abs(rh * w * du) + np.abs(h) * rh ** 3 * m1 / K
    out["dx"] = (scale * d, abs(scale) * size)
    if y is None:
        return out
    c = g * wp
    along, along_size = t * ry * d * y, np.abs(t * ry * y) * size
    if w_post is not None:
        out["dw_post"] = (g[:, 0] * along.sum(axis=1), np.abs(g[:, 0]) * along_size.sum(axis=1))
    if gate is not None:
        out["dgate"] = (wp[:, 0] * along.sum(axis=1), np.abs(wp[:, 0]) * along_size.sum(axis=1))
    S, S_size = (c * d * y).sum(axis=0), (np.abs(c * y) * size).sum(axis=0)
    if token_gate is not None:
        out["dtoken_gate"] = (S * ry[0], S_size * np.abs(ry[0]))
    if w_post is not None:
        out["dy"] = (t * (c * ry * d - y * ry ** 3 * S / K),
                     np.abs(t) * (np.abs(c * ry) * size + np.abs(y * ry ** 3) * S_size / K))
    else:
        out["dy"] = (t * c * d, np.abs(t * c) * size)
    return out
