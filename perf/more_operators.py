"""Operators of a transformer's dense parts beside its compressed layers, as a program calls them: layers that stay in 16 bits,
with what follows the product in its epilogue, and layer norms, both with their gradients.

A case names one operator (`kind`) and its sizes:

  linear           Y = act(W X + bias) + residual, with Z = W X + bias beside it where a training step keeps it
  linear_grad      from dY: dZ = dY act'(Z), dX = W^T dZ, dW = dZ X^T and dbias = the sum of dZ over the tokens
  layer_norm       u = (x - mean) rstd w + b over a token's channels, with mean and rstd
  layer_norm_grad  from du: dx = dh + the gradient through the norm, dw and db = sums over the tokens

Matrices are channels x tokens, row-major, as this package's products take them; layers and token counts are those of
hinm_synth.py (encoder layers, MLP layers for decoding and prefill, square layers, large layer), ragged counts beside even
ones; `draw` spreads over the same ranges, from one token on.

With `own` false everything is computed in elementary torch operations in 32 bits.
"""
import math

import torch

own = False

TORCH_DTYPE = {"f16": torch.float16, "bf16": torch.bfloat16}
DEV = "cuda:0"
EPS = 1e-5
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")


def _library():
    import paper_2407_20496_amd as hinm
    return hinm


def _linear(kind, M, K, N, dtype, act="none", bias=True, residual=False, keep=False, name=None):
    c = {"kind": kind, "M": M, "K": K, "N": N, "dtype": dtype, "act": act, "bias": bias, "residual": residual, "keep": keep}
    return {"name": name, **c} if name else c


def _norm(kind, K, N, dtype, stream=False, name=None):
    c = {"kind": kind, "M": 0, "K": K, "N": N, "dtype": dtype, "stream": stream}
    return {"name": name, **c} if name else c


def listed():
    return [
        # the smallest call: a small head on four tokens, where only the call itself counts
        _linear("linear", 256, 256, 4, "f16", act="relu", name="linear_tiny"),
        # decoding one token through an up-projection: bound by the weights
        _linear("linear", 11008, 4096, 1, "bf16", act="silu", name="linear_1_token"),
        # decoding a batch of 16 sequences through a down-projection, back onto the residual stream
        _linear("linear", 4096, 11008, 16, "bf16", residual=True, name="linear_16_tokens"),
        # an attention block's output projection in an encoder, 32 sequences of 128 tokens
        _linear("linear", 768, 768, 4096, "f16", residual=True, name="linear_encoder"),
        # a training step's up-projection, ragged token count, Z kept for the gradients
        _linear("linear", 11008, 4096, 1571, "bf16", act="gelu", keep=True, name="linear_train_ragged"),
        # the largest product: bound by arithmetic
        _linear("linear", 16384, 16384, 8192, "bf16", act="relu", name="linear_large"),
        # training step of a square layer
        _linear("linear_grad", 4096, 4096, 2048, "bf16", act="gelu", name="linear_grad_square"),
        # training step of an encoder's projection
        _linear("linear_grad", 768, 768, 4096, "f16", name="linear_grad_encoder"),
        # decoding one token: ahead of a layer
        _norm("layer_norm", 4096, 1, "bf16", name="layer_norm_1_token"),
        # prefill, ragged token count
        _norm("layer_norm", 4096, 2047, "bf16", name="layer_norm_ragged"),
        # training step of an encoder, the norm ahead of a block: the residual stream's gradient is added
        _norm("layer_norm_grad", 768, 4096, "f16", stream=True, name="layer_norm_grad_encoder"),
        # training step of a wide layer, ragged token count
        _norm("layer_norm_grad", 16384, 1000, "bf16", name="layer_norm_grad_wide"),
    ]


# ---- drawn cases ----------------------------------------------------------------------------------

def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _channels(rng, lo, hi):
    """Channel counts: mostly whole groups of 32, some whole groups of 8, some odd."""
    c, r = _log(rng, lo, hi), rng.random()
    return max(32, c // 32 * 32) if r < 0.6 else max(8, c // 8 * 8) if r < 0.8 else c


def _tokens(rng, hi):
    """Token counts over 1..hi: single tokens, small batches, ragged and even large ones."""
    if rng.random() < 0.15:
        return 1
    n = _log(rng, 2, hi)
    return n if rng.random() < 0.6 or n < 16 else n // 16 * 16


def draw(rng):
    kind = rng.choices(["linear", "linear_grad", "layer_norm", "layer_norm_grad"], [45, 25, 15, 15])[0]
    dtype = rng.choice(["f16", "bf16"])
    if kind == "linear":
        return _linear(kind, _channels(rng, 128, 16384), _channels(rng, 128, 16384), _tokens(rng, 8192), dtype,
                       act=rng.choice(ACTS), bias=rng.random() < 0.7, residual=rng.random() < 0.4, keep=rng.random() < 0.3)
    if kind == "linear_grad":
        return _linear(kind, _channels(rng, 128, 11008), _channels(rng, 128, 8192), _tokens(rng, 4096), dtype,
                       act=rng.choice(ACTS), bias=rng.random() < 0.7)
    return _norm(kind, _channels(rng, 64, 16384), _tokens(rng, 8192), dtype,
                 stream=kind == "layer_norm_grad" and rng.random() < 0.5)


# ---- preparation ------------------------------------------------------------------------------------

def _ld(N):
    return N if N == 1 else (N + 7) // 8 * 8


def _matrix(K, N, dtype, gen, spread=0.0, shift=0.0):
    """[K][N] in rows of whole groups of eight, N(shift, 1) times a channel's own size (e ** N(0, spread ** 2))."""
    X = torch.zeros((K, _ld(N)), dtype=TORCH_DTYPE[dtype], device=DEV)
    size = torch.exp(spread * torch.randn(K, 1, device=DEV, generator=gen)) if spread else 1.0
    X[:, :N] = ((torch.randn(K, N, device=DEV, generator=gen) + shift) * size).to(TORCH_DTYPE[dtype])
    return X


def _inputs(case, seed):
    """The inputs alone, from the seed."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    kind, M, K, N, dtype = (case[k] for k in ("kind", "M", "K", "N", "dtype"))
    if kind in ("linear", "linear_grad"):
        s = {"W": (torch.randn(M, K, device=DEV, generator=gen) / math.sqrt(K)).to(TORCH_DTYPE[dtype]),
             "X": _matrix(K, N, dtype, gen, 0.3), "bias": None, "residual": None, "Z": None}
        if kind == "linear":
            if case["bias"]:
                s["bias"] = 0.5 * torch.randn(M, device=DEV, generator=gen)
            if case["residual"]:
                s["residual"] = _matrix(M, N, dtype, gen, 0.5)
            return s
        if case["act"] != "none":
            s["Z"] = _matrix(M, N, dtype, gen, 0.3)
        s["dY"] = _matrix(M, N, dtype, gen, 0.3)
        return s
    s = {"w": 1.0 + 0.2 * torch.randn(K, device=DEV, generator=gen), "b": None, "dh": None}
    # a residual stream has channels far larger than the rest, and tokens with a mean
    s["x"] = _matrix(K, N, dtype, gen, 0.8, 0.3)
    if kind == "layer_norm":
        s["b"] = 0.2 * torch.randn(K, device=DEV, generator=gen)
        return s
    s["du"] = _matrix(K, N, dtype, gen)
    if case["stream"]:
        s["dh"] = _matrix(K, N, dtype, gen)
    x = s["x"][:, :N].double()
    mean = x.mean(0)
    s["mean"], s["rstd"] = mean.float(), torch.rsqrt((x - mean).square().mean(0) + EPS).float()
    return s


def prepare(case, seed):
    kind, M, K, N, dtype = (case[k] for k in ("kind", "M", "K", "N", "dtype"))
    s = {**case, "ld": _ld(N), **_inputs(case, seed)}
    if not own:
        return s
    hinm = _library()
    matrix = lambda rows: torch.empty((rows, _ld(N)), dtype=TORCH_DTYPE[dtype], device=DEV)
    f32 = lambda n: torch.empty(n, dtype=torch.float32, device=DEV)
    if kind == "linear":
        s["Y"], s["Z"] = matrix(M), matrix(M) if case["keep"] else None
        nbytes = hinm.hinm_linear_workspace(M, K, N)
    elif kind == "linear_grad":
        s["dX"], s["dW"] = matrix(K), torch.empty((M, K), dtype=TORCH_DTYPE[dtype], device=DEV)
        s["dbias"] = f32(M) if case["bias"] else None
        nbytes = hinm.hinm_linear_grad_workspace(M, K, N)
    elif kind == "layer_norm":
        s["u"], s["mean"], s["rstd"] = matrix(K), f32(N), f32(N)
        nbytes = hinm.hinm_layer_norm_workspace(K, N)
    else:
        s["dx"], s["dw"], s["db"] = matrix(K), f32(K), f32(K)
        nbytes = hinm.hinm_layer_norm_grad_workspace(K, N)
    s["workspace"] = torch.empty(max(nbytes, 1), dtype=torch.uint8, device=DEV), nbytes
    return s


# ---- the plain forms --------------------------------------------------------------------------------

def _activation(v, act):
    if act == "relu":
        return torch.relu(v)
    if act == "gelu":
        return v * 0.5 * (1 + torch.erf(v * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return v * 0.5 * (1 + torch.tanh(math.sqrt(2 / math.pi) * (v + 0.044715 * v * v * v)))
    if act == "silu":
        return v * torch.sigmoid(v)
    return v


def _slope(v, act):
    if act == "relu":
        return (v > 0).to(v.dtype)
    if act == "gelu":
        return 0.5 * (1 + torch.erf(v * math.sqrt(0.5))) + v * torch.exp(-0.5 * v * v) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        t = torch.tanh(math.sqrt(2 / math.pi) * (v + 0.044715 * v * v * v))
        return 0.5 * (1 + t) + 0.5 * v * (1 - t * t) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * v * v)
    s = torch.sigmoid(v)
    return s * (1 + v * (1 - s))


def _plain(s):
    kind, K, N, dtype = s["kind"], s["K"], s["N"], TORCH_DTYPE[s["dtype"]]
    if kind == "linear":
        Z = s["W"].float() @ s["X"][:, :N].float()
        if s["bias"] is not None:
            Z = Z + s["bias"][:, None]
        Y = _activation(Z, s["act"])
        if s["residual"] is not None:
            Y = Y + s["residual"][:, :N].float()
        return [Y.to(dtype), Z.to(dtype)] if s["keep"] else [Y.to(dtype)]
    if kind == "linear_grad":
        dZ = s["dY"][:, :N].float()
        if s["Z"] is not None:
            dZ = dZ * _slope(s["Z"][:, :N].float(), s["act"])
        dX, dW = s["W"].float().t() @ dZ, dZ @ s["X"][:, :N].float().t()
        return [dX.to(dtype), dW.to(dtype)] + ([dZ.sum(1)] if s["bias"] else [])
    x = s["x"][:, :N].float()
    if kind == "layer_norm":
        mean = x.mean(0)
        d = x - mean
        rstd = torch.rsqrt(d.square().mean(0) + EPS)
        return [(d * rstd * s["w"][:, None] + s["b"][:, None]).to(dtype), mean, rstd]
    du = s["du"][:, :N].float()
    xn = (x - s["mean"]) * s["rstd"]
    g = du * s["w"][:, None]
    dx = s["rstd"] * (g - g.mean(0) - xn * (g * xn).mean(0))
    if s["dh"] is not None:
        dx = dx + s["dh"][:, :N].float()
    return [dx.to(dtype), (du * xn).sum(1), du.sum(1)]


# ---- one pass ---------------------------------------------------------------------------------------

def run(s):
    if not own:
        return _plain(s)
    hinm = _library()
    kind, M, K, N, dtype, ld = s["kind"], s["M"], s["K"], s["N"], s["dtype"], s["ld"]
    if kind in ("linear", "linear_grad"):
        flags = {"none": 0, "relu": hinm.EPI_RELU, "gelu": hinm.EPI_GELU, "gelu_tanh": hinm.EPI_GELU_TANH,
                 "silu": hinm.EPI_SILU}[s["act"]]
    if kind == "linear":
        hinm.hinm_linear(M, K, N, dtype, s["W"], K, s["X"], ld, s["bias"], s["residual"], ld, s["Z"], s["Y"], ld, flags,
                         *s["workspace"])
        return [s["Y"][:, :N]] + ([s["Z"][:, :N]] if s["keep"] else [])
    if kind == "linear_grad":
        hinm.hinm_linear_grad(M, K, N, dtype, s["W"], K, s["X"], ld, s["Z"], s["dY"], ld, s["dX"], s["dW"], s["dbias"], flags,
                              *s["workspace"])
        return [s["dX"][:, :N], s["dW"]] + ([s["dbias"]] if s["bias"] else [])
    if kind == "layer_norm":
        hinm.hinm_layer_norm(K, N, dtype, EPS, s["x"], ld, s["w"], s["b"], s["u"], ld, s["mean"], s["rstd"], *s["workspace"])
        return [s["u"][:, :N], s["mean"], s["rstd"]]
    hinm.hinm_layer_norm_grad(K, N, dtype, s["x"], ld, s["w"], s["mean"], s["rstd"], s["du"], ld, s["dh"], s["dx"], s["dw"],
                              s["db"], *s["workspace"])
    return [s["dx"][:, :N], s["dw"], s["db"]]


# ---- from the definition, in 64 bits ------------------------------------------------------------------

def _rate64(z, act):
    """(act(z) / z, act'(z)) of float64 values."""
    if act == "none":
        return torch.ones_like(z), torch.ones_like(z)
    if act == "relu":
        on = torch.where(z > 0, 1.0, 0.0).to(z.dtype)
        return on, on
    if act == "gelu":               # z times the normal distribution's probability of less than z
        p = torch.special.erfc(z / -(2 ** 0.5)) / 2
        return p, p + z * torch.exp(z.square() / -2) / (2 * math.pi) ** 0.5
    # z sigmoid(q(z)): q = z, or twice the argument of tanh
    c = 2 * (2 / math.pi) ** 0.5
    q, slope = (z, 1.0) if act == "silu" else (c * (z + 0.044715 * z.pow(3)), c * (1 + 0.134145 * z.square()))
    p = 1 / (1 + torch.exp(-q))
    return p, p + z * p * (1 / (1 + torch.exp(q))) * slope


def exact(case, seed):
    kind, K, N = case["kind"], case["K"], case["N"]
    i = _inputs(case, seed)
    if kind == "linear":
        X = i["X"][:, :N].double()
        Y, Z = [], []
        for r in range(0, case["M"], 4096):
            z = torch.mm(i["W"][r:r + 4096].double(), X)
            if i["bias"] is not None:
                z += i["bias"][r:r + 4096].double().unsqueeze(1)
            y = z * _rate64(z, case["act"])[0]
            if i["residual"] is not None:
                y += i["residual"][r:r + 4096, :N].double()
            Y.append(y)
            Z.append(z if case["keep"] else None)
        return [torch.cat(Y)] + ([torch.cat(Z)] if case["keep"] else [])
    if kind == "linear_grad":
        g = i["dY"][:, :N].double()
        if i["Z"] is not None:
            g = g * _rate64(i["Z"][:, :N].double(), case["act"])[1]
        out = [torch.mm(i["W"].double().t(), g), torch.mm(g, i["X"][:, :N].double().t())]
        return out + ([torch.mv(g, torch.ones(N, dtype=g.dtype, device=DEV))] if case["bias"] else [])
    x, w = i["x"][:, :N].double(), i["w"].double().unsqueeze(1)
    if kind == "layer_norm":
        mean = x.sum(0) / K
        root = ((x.pow(2).sum(0) / K - mean.pow(2)) + EPS).pow(-0.5)
        return [x * (w * root) + (i["b"].double().unsqueeze(1) - w * (mean * root)), mean, root]
    # with t = x - mean and r = rstd as they are given, the gradient of r t w applied to du
    du, r = i["du"][:, :N].double(), i["rstd"].double()
    t = x - i["mean"].double()
    along = (w * du * t).sum(0)
    dx = r * w * du - r / K * (w * du).sum(0) - r.pow(3) / K * along * t
    if i["dh"] is not None:
        dx += i["dh"][:, :N].double()
    return [dx, torch.mv(du * t, r), du.sum(1)]


# ---- what a pass cannot do without --------------------------------------------------------------------

def work(case):
    kind, M, K, N = (case[k] for k in ("kind", "M", "K", "N"))
    if kind == "linear":
        return {"bytes": 2 * (M * K + K * N + M * N * (1 + case["residual"] + case["keep"])) + 4 * M * case["bias"],
                "flops": 2 * M * K * N}
    if kind == "linear_grad":
        return {"bytes": 2 * (2 * M * K + 2 * K * N + M * N * (1 + (case["act"] != "none"))) + 4 * M * case["bias"],
                "flops": 4 * M * K * N}
    if kind == "layer_norm":
        return {"bytes": 4 * K * N + 8 * K + 8 * N, "flops": 8 * K * N}
    return {"bytes": 2 * K * N * (3 + case["stream"]) + 12 * K + 8 * N, "flops": 14 * K * N}
