"""Dense layers with their epilogue, layer norm, and the gradients of both, in float64 from the formulas (include/hinm.h).

Arrays are numpy float64, channels x tokens.  Nothing here is shared with the library."""
import math

import numpy as np

ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")
_erf = np.vectorize(math.erf, otypes=[np.float64])
_erfc = np.vectorize(math.erfc, otypes=[np.float64])


def _sigmoid(q):
    e = np.exp(-np.abs(q))
    return np.where(q >= 0, 1 / (1 + e), e / (1 + e))


def act(z, name):
    if name == "none":
        return z
    if name == "relu":
        return np.where(z > 0, z, 0.0)
    if name == "gelu":
        return z * _erfc(-z / math.sqrt(2)) / 2
    if name == "gelu_tanh":
        return z * _sigmoid(2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))
    return z * _sigmoid(z)


def slope(z, name):
    if name == "none":
        return np.ones_like(z)
    if name == "relu":
        return (z > 0).astype(np.float64)
    if name == "gelu":
        return _erfc(-z / math.sqrt(2)) / 2 + z * np.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        c = 2 * math.sqrt(2 / math.pi)
        s = _sigmoid(c * (z + 0.044715 * z ** 3))
        return s + z * s * (1 - s) * c * (1 + 3 * 0.044715 * z * z)
    s = _sigmoid(z)
    return s * (1 + z * (1 - s))


def linear(W, X, bias=None, residual=None, name="none"):
    """(Y, Z)"""
    Z = W @ X
    if bias is not None:
        Z = Z + bias[:, None]
    Y = act(Z, name)
    return (Y if residual is None else Y + residual), Z


def linear_grad(W, X, Z, dY, name="none"):
    """(dX, dW, dbias, dZ)"""
    dZ = dY if name == "none" else dY * slope(Z, name)
    return W.T @ dZ, dZ @ X.T, dZ.sum(1), dZ


def layer_norm(x, w, b, eps):
    """(u, mean, rstd)"""
    mean = x.mean(0)
    rstd = 1 / np.sqrt(((x - mean) ** 2).mean(0) + eps)
    u = (x - mean) * rstd
    if w is not None:
        u = u * w[:, None]
    return (u if b is None else u + b[:, None]), mean, rstd


def layer_norm_grad(x, w, mean, rstd, du, dh=None):
    """(dx, dw, db)"""
    xn = (x - mean) * rstd
    g = du if w is None else du * w[:, None]
    dx = rstd * (g - g.mean(0) - xn * (g * xn).mean(0))
    return (dx if dh is None else dx + dh), (du * xn).sum(1), du.sum(1)
