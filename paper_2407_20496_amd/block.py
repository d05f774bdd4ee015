"""A transformer's feed-forward block between its norms, on channels x tokens matrices, over the C-ABI entry points.

    h = a x + gate . norm(layers(u)) w_post        u_next = norm(h) w_next

Layers come in either compressed form, prepared HiNM layers (`Layer`, run by hinm_chain) or 4-bit ones (`Mx4Layer`, run by
hinm_mx4_linear), or as they were before (`DenseLayer`, run by hinm_linear, with bias and activation).  This module holds buffers
and hands arrays from one call to the next; everything that is computed runs in
the library's kernels, on the current stream.  PyTorch is used for device memory only.

    up, down = mx4_layer(W_up, flags=hb.EPI_RELU), mx4_layer(W_down)
    block = FeedForward([up, down], tokens, w_post, w_next=w_next_block)
    u = block_input(x, w_pre, tokens)
    x, u = block(x, u)            # and on to the next block with these

An encoder's block with a layer norm ahead of it, for inference and for a training step (dense layers):

    ffn = LayerNormFeedForward([dense_layer(W_up, b_up, hb.EPI_GELU), dense_layer(W_down, b_down)], tokens, w, b)
    h = ffn(x)                                  # x + down(gelu(up(layer_norm(x))))
    dx, gradients = ffn.backward(x, dh)
"""
from __future__ import annotations

from dataclasses import dataclass
from typing import Optional, Sequence, Tuple, Union

import torch

from . import binding as hb


@dataclass
class Mx4Layer:
    """Weights [M][K] in microscaled 4-bit form; flags as for hinm_mx4_linear (EPI_RELU between layers;
    OUT_F32 is not for layers of a block)."""
    M: int
    K: int
    dtype: object
    codes: torch.Tensor
    scales: torch.Tensor
    flags: int = 0


@dataclass
class DenseLayer:
    """16-bit weights [M][K] in rows of any pitch, a float32 bias [M] or none; flags: an activation of hinm_linear's."""
    M: int
    K: int
    dtype: object
    W: torch.Tensor
    bias: Optional[torch.Tensor] = None
    flags: int = 0


_TORCH_DTYPE = {hb.F16: torch.float16, hb.BF16: torch.bfloat16}


def _row_pitch(t: torch.Tensor, what: str) -> int:
    """Leading dimension of a 16-bit matrix whose rows of consecutive values lie apart; ValueError for anything else (the
    library is told addresses and cannot see it)."""
    if t.dim() != 2 or t.dtype not in _TORCH_DTYPE.values():
        raise ValueError(f"{what}: a float16 or bfloat16 matrix wanted, not {t.dtype} {list(t.shape)}")
    rows, cols = t.shape
    if (cols > 1 and t.stride(1) != 1) or (rows > 1 and t.stride(0) < cols):
        raise ValueError(f"{what}: rows of consecutive values apart from each other wanted, not strides {t.stride()}")
    return t.stride(0) if rows > 1 else cols


def _pitch(t: torch.Tensor, what: str, tokens: int, K: Optional[int] = None, dtype=None, device=None) -> int:
    """... of a [K][>= tokens] one; one token may be a vector."""
    if K is not None and t.dim() == 2 and t.dtype is dtype and t.device == device:  # a step pays for this: 0.8 us here, 2.1 below
        (rows, cols), (ld, step) = t.shape, t.stride()
        if rows == K > 1 and cols >= tokens and ld >= cols and step == 1:
            return ld
    if t.dim() == 1 and tokens == 1:
        t = t.unsqueeze(1)
    ld = _row_pitch(t, what)
    if t.shape[1] < tokens or (K is not None and t.shape[0] != K):
        raise ValueError(f"{what}: [{'channels' if K is None else K}][at least {tokens}] wanted, not {list(t.shape)}")
    if (dtype is not None and t.dtype != dtype) or (device is not None and t.device != device):
        raise ValueError(f"{what}: {dtype} on {device} wanted, not {t.dtype} on {t.device}")
    return ld


def _place(t: torch.Tensor) -> Tuple[int, int, int, int]:
    """Where a block's buffer lies: address, bytes, rows, leading dimension."""
    return t.data_ptr(), t.nbytes, t.shape[0], t.stride(0)


def _is_own(t: torch.Tensor, ld: int, what: str, tokens: int, own: Tuple[int, int, int, int]) -> bool:
    """Whether an array that _pitch took is a block's buffer itself, which lies at `own`; ValueError where it shares memory with it
    in another way, so that one would be written while the other is still read.  0.3 us of a call."""
    at, nbytes, rows, pitch = own
    distance = t.data_ptr() - at
    if distance >= nbytes or distance <= -2 * ((rows - 1) * ld + tokens):
        return False
    if distance or (rows > 1 and ld != pitch):
        raise ValueError(f"{what}: overlaps the block's own buffer")
    return True


def _factors(t: Optional[torch.Tensor], what: str, n: int, device) -> None:
    """n float32 values or more, one after the other, or none at all."""
    if t is not None and (t.dtype is not torch.float32 or t.numel() < n or not t.is_contiguous() or t.device != device):
        raise ValueError(f"{what}: {n} consecutive float32 on {device} wanted, not {list(t.shape)} {t.dtype} on {t.device}")


def mx4_form(rows: int, length: int, device) -> Tuple[torch.Tensor, torch.Tensor]:
    """Memory for codes and scales of `rows` rows of `length` values."""
    cb, sb = hb.hinm_mx4_sizes(rows, length)
    return torch.empty(cb, dtype=torch.uint8, device=device), torch.empty(sb, dtype=torch.uint8, device=device)


def mx4_layer(W: torch.Tensor, flags: int = 0) -> Mx4Layer:
    """Dense 16-bit weights [M][K] (rows may lie apart) to a 4-bit layer."""
    ld = _row_pitch(W, "weights")
    M, K = W.shape
    codes, scales = mx4_form(M, K, W.device)
    hb.hinm_mx4_quantize(M, K, W.dtype, W, ld, hb.MX4_ROWS, codes, scales)
    return Mx4Layer(M, K, W.dtype, codes, scales, flags)


_ACTIVATIONS = (0, hb.EPI_RELU, hb.EPI_GELU, hb.EPI_GELU_TANH, hb.EPI_SILU)


def _check_activation(flags: int) -> None:
    if flags not in _ACTIVATIONS:
        raise ValueError(f"flags: one activation or none wanted, not {flags:#x}")


def dense_layer(W: torch.Tensor, bias: Optional[torch.Tensor] = None, flags: int = 0) -> DenseLayer:
    """A layer of the weights as they are (kept, not copied); flags: one activation or none."""
    _row_pitch(W, "weights")
    M, K = W.shape
    _factors(bias, "bias", M, W.device)
    _check_activation(flags)
    return DenseLayer(M, K, W.dtype, W, bias, flags)


def mx4_linear_grad(W: torch.Tensor, X: torch.Tensor, dY: torch.Tensor, tokens: Optional[int] = None,
                    want_input: bool = True, want_weights: bool = True):
    """Gradients of Y = W X where every product is taken on 4-bit operands, each quantised along the axis that is summed over
    and rounded as if the quantisation were not there (straight through): (dX like X, dW float32 [M][K]).
    W [M][K], X [K][>= tokens], dY [M][>= tokens] of one type on one device, in rows of any pitch (others raise ValueError);
    `tokens` columns are in use (all of X's where it is not given), and dX's columns beyond them are left as they are allocated."""
    ld_w = _row_pitch(W, "W")
    M, K = W.shape
    dev, dtype = W.device, W.dtype
    N = tokens if tokens is not None else X.shape[-1]
    ld_x, ld_dy = _pitch(X, "X", N, K, dtype, dev), _pitch(dY, "dY", N, M, dtype, dev)
    dX = dW = None
    if want_input:
        across_w, across_dy = mx4_form(K, M, dev), mx4_form(N, M, dev)
        hb.hinm_mx4_quantize(M, K, dtype, W, ld_w, hb.MX4_COLUMNS, *across_w)
        hb.hinm_mx4_quantize(M, N, dtype, dY, ld_dy, hb.MX4_COLUMNS, *across_dy)
        dX = torch.empty(X.shape, dtype=dtype, device=dev)
        hb.hinm_mx4_product(K, N, M, dtype, *across_w, *across_dy, dX, X.shape[1])
    if want_weights:
        along_dy, along_x = mx4_form(M, N, dev), mx4_form(K, N, dev)
        hb.hinm_mx4_quantize(M, N, dtype, dY, ld_dy, hb.MX4_ROWS, *along_dy)
        hb.hinm_mx4_quantize(K, N, dtype, X, ld_x, hb.MX4_ROWS, *along_x)
        dW = torch.empty((M, K), dtype=torch.float32, device=dev)
        hb.hinm_mx4_product(M, K, N, dtype, *along_dy, *along_x, dW, K, hb.OUT_F32)
    return dX, dW


def leading_dimension(tokens: int) -> int:
    """Columns of a buffer for `tokens` tokens: whole 16-byte pieces, or one alone."""
    return tokens if tokens == 1 else (tokens + 7) // 8 * 8


def _workspace(nbytes: int, device) -> torch.Tensor:
    return torch.empty(max(nbytes, 1), dtype=torch.uint8, device=device)


def block_input(x: torch.Tensor, w_pre: torch.Tensor, tokens: int, eps: float = 1e-6) -> torch.Tensor:
    """u = norm(x) w_pre: what the first block's layers take.  x [K][>= tokens] 16-bit, in rows of any pitch; u has x's shape,
    contiguous (a FeedForward takes it where that is [K][leading_dimension(tokens)])."""
    ld = _pitch(x, "x", tokens)
    K = x.shape[0]
    _factors(w_pre, "w_pre", K, x.device)
    u = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    nbytes = hb.hinm_block_norm_workspace(K, tokens)
    hb.hinm_block_norm(K, tokens, x.dtype, 1.0, eps, x, None, None, None, None, w_pre, None, ld, u, x.shape[1], None, None,
                       _workspace(nbytes, x.device), nbytes)
    return u


def _check_layers(layers: Sequence[DenseLayer], device) -> None:
    """What the library cannot see of dense layers: their arrays' shapes, types and places, and that their results go to 16-bit
    buffers."""
    for l in layers:
        _check_activation(l.flags)
        _row_pitch(l.W, "weights")
        if list(l.W.shape) != [l.M, l.K] or l.W.dtype != _TORCH_DTYPE[hb._dtype_code(l.dtype)] or l.W.device != device:
            raise ValueError(f"weights: {l.dtype} [{l.M}][{l.K}] on {device} wanted, not {l.W.dtype} {list(l.W.shape)} on {l.W.device}")
        _factors(l.bias, "bias", l.M, device)


class FeedForward:
    """One block for a fixed number of tokens: its layers, norms and buffers.

    x is [K][>= tokens] in rows of any pitch, u [K][>= tokens] in rows of leading_dimension(tokens), which is the pitch of the
    block's own buffers too; both of the layers' type, on the block's device.  Other arrays raise ValueError."""

    def __init__(self, layers: Sequence[Union[Mx4Layer, DenseLayer, hb.Layer]], tokens: int, w_post: Optional[torch.Tensor],
                 gate: Optional[torch.Tensor] = None, w_next: Optional[torch.Tensor] = None, residual_scale: float = 1.0,
                 eps: float = 1e-6, device="cuda"):
        layers = list(layers)
        if not layers or any(a.M != b.K for a, b in zip(layers, layers[1:])) or layers[-1].M != layers[0].K:
            raise ValueError("layers must follow one another and lead back to the block's channels")
        self.in_4_bits, self.dense = (all(isinstance(l, form) for l in layers) for form in (Mx4Layer, DenseLayer))
        if not (self.in_4_bits or self.dense) and any(isinstance(l, (Mx4Layer, DenseLayer)) for l in layers):
            raise ValueError("one block's layers come in one form")
        if len({hb._dtype_code(l.dtype) for l in layers}) > 1:
            raise ValueError("one block's layers have one type")
        if any(l.flags & hb.OUT_F32 for l in layers):
            raise ValueError("flags: OUT_F32 is not for a block, whose buffers are 16-bit")
        self.layers, self.tokens, self.ld = layers, tokens, leading_dimension(tokens)
        self.w_post, self.gate, self.w_next = w_post, gate, w_next
        self.residual_scale, self.eps = residual_scale, eps
        self.K, self.dtype = layers[0].K, layers[0].dtype
        new = lambda rows: torch.empty((rows, self.ld), dtype=_TORCH_DTYPE[hb._dtype_code(self.dtype)], device=device)
        self.y = new(self.K)
        self._y_place = _place(self.y)
        for what, t in (("w_post", w_post), ("gate", gate), ("w_next", w_next)):
            _factors(t, what, self.K, self.y.device)
        for l in layers if self.in_4_bits else ():
            for t, n in zip((l.codes, l.scales), hb.hinm_mx4_sizes(l.M, l.K)):
                if t.dtype != torch.uint8 or t.numel() < n or not t.is_contiguous() or t.device != self.y.device:
                    raise ValueError(f"weights: {n} bytes on {self.y.device} wanted, not {t.dtype} {list(t.shape)} on {t.device}")
        if self.dense:
            _check_layers(layers, self.y.device)
            self.ldw = [_row_pitch(l.W, "weights") for l in layers]
        if self.in_4_bits or self.dense:
            self.between = [new(l.M) for l in layers[:-1]]
            bytes_of = hb.hinm_mx4_linear_workspace if self.in_4_bits else hb.hinm_linear_workspace
            self.scratch_bytes = max(bytes_of(l.M, l.K, tokens) for l in layers)
        else:
            self.scratch_bytes = hb.hinm_chain_sizes(layers, tokens)
        self.scratch = _workspace(self.scratch_bytes, device)
        self.norm_bytes = hb.hinm_block_norm_workspace(self.K, tokens)
        self.norm_workspace = _workspace(self.norm_bytes, device)

    def run_layers(self, u: torch.Tensor) -> torch.Tensor:
        """y = layers(u), in the block's own buffer."""
        N, ld = self.tokens, self.ld
        if _pitch(u, "u", N, self.K, self.y.dtype, self.y.device) != ld:
            raise ValueError(f"u: rows of {ld} = leading_dimension({N}) values wanted, not strides {u.stride()}")
        if _is_own(u, ld, "u", N, self._y_place) and len(self.layers) == 1:
            raise ValueError("u: one layer cannot write over its input")
        if self.dense:
            for l, ldw, out in zip(self.layers, self.ldw, self.between + [self.y]):
                hb.hinm_linear(l.M, l.K, N, l.dtype, l.W, ldw, u, ld, l.bias, None, 0, None, out, ld, l.flags, self.scratch,
                               self.scratch_bytes)
                u = out
            return u
        if not self.in_4_bits:
            hb.hinm_chain(self.layers, N, u, ld, self.y, ld, self.scratch, self.scratch_bytes)
            return self.y
        for l, out in zip(self.layers, self.between + [self.y]):
            hb.hinm_mx4_linear(l.M, l.K, N, l.dtype, l.codes, l.scales, u, ld, out, ld, l.flags, self.scratch,
                               self.scratch_bytes)
            u = out
        return u

    def __call__(self, x: torch.Tensor, u: torch.Tensor, token_gate: Optional[torch.Tensor] = None):
        """(h, u_next) in place of (x, u); u_next is u untouched where no norm follows."""
        ld_stream = _pitch(x, "x", self.tokens, self.K, self.y.dtype, self.y.device)
        _factors(token_gate, "token_gate", self.tokens, self.y.device)
        y = self.run_layers(u)
        hb.hinm_block_norm(self.K, self.tokens, self.dtype, self.residual_scale, self.eps, x, y, self.w_post, self.gate,
                           token_gate, self.w_next, x, ld_stream, u, self.ld, None, None, self.norm_workspace, self.norm_bytes)
        return x, u


class LayerNormFeedForward:
    """h = x + layers(layer_norm(x) w + b) for a fixed number of tokens, and its gradients: dense layers, buffers of one step.

    x and dh are [K][>= tokens] in rows of one pitch, of the layers' type on the block's device; other arrays raise ValueError.  A
    step of training is a call and then `backward` with the same x; h, dx and the gradients are the block's own buffers, which its
    next call or backward pass overwrites."""

    def __init__(self, layers: Sequence[DenseLayer], tokens: int, w: Optional[torch.Tensor] = None, b: Optional[torch.Tensor] = None,
                 eps: float = 1e-5, device="cuda"):
        layers = list(layers)
        if not layers or not all(isinstance(l, DenseLayer) for l in layers):
            raise ValueError("dense layers wanted")
        if any(a.M != b.K for a, b in zip(layers, layers[1:])) or layers[-1].M != layers[0].K:
            raise ValueError("layers must follow one another and lead back to the block's channels")
        if len({hb._dtype_code(l.dtype) for l in layers}) > 1:
            raise ValueError("one block's layers have one type")
        if layers[-1].flags:
            raise ValueError("the last layer leads back to the stream: without an activation")
        self.layers, self.tokens, self.ld, self.eps = layers, tokens, leading_dimension(tokens), eps
        self.K, self.dtype = layers[0].K, layers[0].dtype
        self.w, self.b = w, b
        new = lambda rows: torch.empty((rows, self.ld), dtype=_TORCH_DTYPE[hb._dtype_code(self.dtype)], device=device)
        f32 = lambda n: torch.empty(n, dtype=torch.float32, device=device)
        self.u = new(self.K)
        self.device = self.u.device
        _check_layers(layers, self.device)
        for what, t in (("w", w), ("b", b)):
            _factors(t, what, self.K, self.device)
        self.h, self.mean, self.rstd = new(self.K), f32(tokens), f32(tokens)
        self._h_place = _place(self.h)
        self.Z = [new(l.M) if l.flags else None for l in layers]
        self.out = [new(l.M) for l in layers[:-1]]
        sizes = [hb.hinm_linear_workspace(l.M, l.K, tokens) for l in layers] + [hb.hinm_layer_norm_workspace(self.K, tokens)]
        self.scratch_bytes = max(sizes)
        self.scratch = _workspace(self.scratch_bytes, device)
        self.ldw = [_row_pitch(l.W, "weights") for l in layers]
        self._backward = self._dx_buffer = None
        self._kept = None  # no call yet; then whether the last one left what a backward pass needs

    def __call__(self, x: torch.Tensor, train: bool = True) -> torch.Tensor:
        """h, in the block's own buffer; with `train` what `backward` needs is kept.  x may be h (a block
        applied again), but then it is overwritten, and nothing is kept."""
        N, ld, ws = self.tokens, self.ld, (self.scratch, self.scratch_bytes)
        ldx = _pitch(x, "x", N, self.K, self.u.dtype, self.device)
        in_place = _is_own(x, ldx, "x", N, self._h_place)
        self._kept = False
        hb.hinm_layer_norm(self.K, N, self.dtype, self.eps, x, ldx, self.w, self.b, self.u, ld, self.mean, self.rstd, *ws)
        into = self.u
        for l, ldw, z, out in zip(self.layers, self.ldw, self.Z, self.out + [self.h]):
            last = out is self.h
            hb.hinm_linear(l.M, l.K, N, l.dtype, l.W, ldw, into, ld, l.bias, x if last else None, ldx, z if train else None, out,
                           ld, l.flags, *ws)
            into = out
        self._kept = train and not in_place
        return self.h

    def backward(self, x: torch.Tensor, dh: torch.Tensor):
        """(dx, gradients): of x, in rows of its pitch; of every layer's W (its type, contiguous) and bias, and of the norm's
        w and b, as a dict of tensors "W0", "bias0", ..., "w", "b" (no entry for what the block does not have).  Ahead of any call it
        makes the call itself; behind one that kept nothing, or one that failed, it raises ValueError.  dh may be dx."""
        N, ld = self.tokens, self.ld
        ldx = _pitch(x, "x", N, self.K, self.u.dtype, self.device)
        if _pitch(dh, "dh", N, self.K, self.u.dtype, self.device) != ldx:
            raise ValueError(f"dh: rows of x's pitch {ldx} wanted, not strides {dh.stride()}")
        dx = self._dx(ldx)
        dx_place = _place(dx)
        if _is_own(x, ldx, "x", N, self._h_place) or _is_own(x, ldx, "x", N, dx_place):
            raise ValueError("x: overwritten by the block")
        _is_own(dh, ldx, "dh", N, dx_place)
        if self._kept is None:
            self(x)
        if not self._kept:
            raise ValueError("the last call kept nothing for a backward pass")
        if self._backward is None:
            new = lambda rows, cols: torch.empty((rows, cols), dtype=self.u.dtype, device=self.device)
            f32 = lambda n: torch.empty(n, dtype=torch.float32, device=self.device)
            g = {}
            for i, l in enumerate(self.layers):
                g[f"W{i}"] = new(l.M, l.K)
                if l.bias is not None:
                    g[f"bias{i}"] = f32(l.M)
            for what, t in (("w", self.w), ("b", self.b)):
                if t is not None:
                    g[what] = f32(self.K)
            nbytes = max([hb.hinm_linear_grad_workspace(l.M, l.K, N) for l in self.layers] + [hb.hinm_layer_norm_grad_workspace(self.K, N)])
            self._backward = g, [new(l.K, ld) for l in self.layers], (_workspace(nbytes, self.device), nbytes)
        g, into, ws = self._backward
        dy, ldy = dh, ldx
        for i, l in reversed(list(enumerate(self.layers))):
            X = self.out[i - 1] if i else self.u
            ldw = self.ldw[i]
            # dX and dW take the pitch of X and W
            dW = g[f"W{i}"] if ldw == l.K else None
            hb.hinm_linear_grad(l.M, l.K, N, l.dtype, l.W, ldw, X, ld, self.Z[i], dy, ldy, into[i], dW, g.get(f"bias{i}"), l.flags, *ws)
            if dW is None:
                hb.hinm_linear_grad(l.M, l.K, N, l.dtype, None, l.K, X, ld, self.Z[i], dy, ldy, None, g[f"W{i}"], None, l.flags, *ws)
            dy, ldy = into[i], ld
        hb.hinm_layer_norm_grad(self.K, N, self.dtype, x, ldx, self.w, self.mean, self.rstd, into[0], ld, dh, dx, g.get("w"), g.get("b"), *ws)
        return dx, g

    def _dx(self, ldx: int) -> torch.Tensor:
        """dx's buffer, in rows of x's pitch as the norm's gradients have it."""
        if self._dx_buffer is None or self._dx_buffer.shape[1] != ldx:
            self._dx_buffer = torch.empty((self.K, ldx), dtype=self.u.dtype, device=self.device)
        return self._dx_buffer
