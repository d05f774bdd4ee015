"""Operators of a transformer's feed-forward block around its compressed layers, as a program calls them.

A case names one operator (`kind`) and its sizes:

  weights4      dense weights [M][K] to microscaled 4-bit form (32 values along a row share a power of two) and back
  tokens4       activations [K][N] to the same form, 32 channels of a token share the power of two, and back
  linear4       Y = act(W4 Q(X)): 4-bit weights that a program keeps, 16-bit activations quantised within the call
  linear4_grad  a training step's two other products: dX = Q(W^T) Q(dY) along the output channels and
                dW = Q(dY) Q(X)^T along the tokens, every operand quantised along the axis it is summed over
  norm          a block's norms on both of its sides: h = a x + gate . token_gate . rmsnorm(y) w_post, u = rmsnorm(h) w_pre
  norm_grad     gradients of the same: of x, y, both weights, the channels' gate and the tokens' gate

Matrices are channels x tokens, row-major, as this package's products take them; layers and token counts are those of
hinm_synth.py (encoder feed-forward layer, MLP layers for decoding and prefill, square layers, large layer), ragged counts
beside even ones; `draw` spreads over the same ranges.

With `own` false everything is computed in elementary torch operations in 32 bits.
"""
import math

import torch

own = False

TORCH_DTYPE = {"f16": torch.float16, "bf16": torch.bfloat16}
DEV = "cuda:0"
EPS = 1e-6


def _library():
    import paper_2407_20496_amd as hinm
    return hinm


def _case(kind, M, K, N, dtype, name=None, **more):
    c = {"kind": kind, "M": M, "K": K, "N": N, "dtype": dtype, **more}
    return {"name": name, **c} if name else c


def _norm(kind, K, N, dtype, post=True, gate=True, token_gate=False, pre=True, scale=1.0, name=None):
    return _case(kind, 0, K, N, dtype, name=name, post=post, gate=gate, token_gate=token_gate, pre=pre, scale=scale)


def listed():
    return [
        # the smallest call: a tiny layer's weights, where only the calls themselves count
        _case("weights4", 256, 256, 0, "f16", name="weights4_tiny"),
        # compressing an up-projection of an MLP block
        _case("weights4", 11008, 4096, 0, "bf16", name="weights4_mlp"),
        # activations of a prefill ahead of a down-projection, ragged token count
        _case("tokens4", 0, 11008, 1571, "bf16", name="tokens4_ragged"),
        # decoding one token through an up-projection: bound by the weights
        _case("linear4", 11008, 4096, 1, "bf16", relu=True, name="linear4_1_token"),
        # decoding a batch of 16 sequences through a down-projection
        _case("linear4", 4096, 11008, 16, "bf16", relu=False, name="linear4_16_tokens"),
        # a square layer, ragged number of tokens, between decoding and prefill
        _case("linear4", 4096, 4096, 1000, "f16", relu=True, name="linear4_1000_tokens"),
        # the largest product: bound by arithmetic
        _case("linear4", 16384, 16384, 8192, "bf16", relu=False, name="linear4_large"),
        # training step of a square layer: gradients of its input and of its weights
        _case("linear4_grad", 4096, 4096, 2048, "bf16", name="linear4_grad_square"),
        # decoding one token: between two blocks of a decoder
        _norm("norm", 4096, 1, "bf16", name="norm_1_token"),
        # prefill, ragged token count, tokens gated one by one
        _norm("norm", 4096, 2047, "bf16", token_gate=True, scale=0.5, name="norm_prefill_ragged"),
        # training step of an encoder's block, 32 sequences of 128 tokens
        _norm("norm_grad", 768, 4096, "f16", token_gate=True, name="norm_grad_encoder"),
        # training step of a wide layer, ragged token count
        _norm("norm_grad", 16384, 1000, "bf16", name="norm_grad_wide"),
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
    kind = rng.choices(["weights4", "tokens4", "linear4", "linear4_grad", "norm", "norm_grad"], [10, 10, 35, 10, 20, 15])[0]
    dtype = rng.choice(["f16", "bf16"])
    if kind == "weights4":
        return _case(kind, _channels(rng, 64, 16384), _channels(rng, 64, 11008), 0, dtype)
    if kind == "tokens4":
        return _case(kind, 0, _channels(rng, 64, 16384), _tokens(rng, 8192), dtype)
    if kind == "linear4":
        return _case(kind, _channels(rng, 128, 16384), _channels(rng, 128, 16384), _tokens(rng, 8192), dtype, relu=rng.random() < 0.5)
    if kind == "linear4_grad":
        return _case(kind, _channels(rng, 128, 11008), _channels(rng, 128, 8192), _tokens(rng, 4096), dtype)
    post = rng.random() < 0.8
    return _norm(kind, _channels(rng, 64, 16384), _tokens(rng, 8192), dtype, post=post, gate=rng.random() < 0.6,
                 token_gate=rng.random() < 0.4, pre=not post or rng.random() < 0.8, scale=rng.choice([1.0, 0.5, 1.75]))


# ---- preparation ------------------------------------------------------------------------------------

def _ld(N):
    return N if N == 1 else (N + 7) // 8 * 8


def _matrix(K, N, dtype, gen, spread=0.0):
    """[K][N] in rows of whole groups of eight, N(0, 1) times a channel's own size (e ** N(0, spread ** 2))."""
    X = torch.zeros((K, _ld(N)), dtype=TORCH_DTYPE[dtype], device=DEV)
    size = torch.exp(spread * torch.randn(K, 1, device=DEV, generator=gen)) if spread else 1.0
    X[:, :N] = (torch.randn(K, N, device=DEV, generator=gen) * size).to(TORCH_DTYPE[dtype])
    return X


def _empty(K, N, dtype):
    return torch.empty((K, _ld(N)), dtype=TORCH_DTYPE.get(dtype, dtype), device=DEV)


def _weights(M, K, dtype, gen):
    return (torch.randn(M, K, device=DEV, generator=gen) * 0.02).to(TORCH_DTYPE[dtype])


def _buffers4(rows, length):
    """Codes and scales of `rows` rows of `length` values."""
    cb, sb = _library().hinm_mx4_sizes(rows, length)
    return (torch.empty(cb, dtype=torch.uint8, device=DEV), torch.empty(sb, dtype=torch.uint8, device=DEV))


def _workspace(nbytes):
    return torch.empty(max(int(nbytes), 1), dtype=torch.uint8, device=DEV), int(nbytes)


def _inputs(case, seed):
    """The inputs alone, from the seed."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    kind, M, K, N, dtype = (case[k] for k in ("kind", "M", "K", "N", "dtype"))
    if kind == "weights4":
        return {"W": _weights(M, K, dtype, gen)}
    if kind == "tokens4":
        return {"X": _matrix(K, N, dtype, gen, 0.5)}
    if kind == "linear4":
        return {"W": _weights(M, K, dtype, gen), "X": _matrix(K, N, dtype, gen, 0.5)}
    if kind == "linear4_grad":
        return {"W": _weights(M, K, dtype, gen), "X": _matrix(K, N, dtype, gen, 0.5), "dY": _matrix(M, N, dtype, gen, 0.5)}
    s = {"w_post": None, "w_pre": None, "gate": None, "token_gate": None}
    around_one = lambda n: 1.0 + 0.2 * torch.randn(n, device=DEV, generator=gen)
    if case["post"]:
        s["w_post"] = around_one(K)
    if case["gate"]:
        s["gate"] = 0.5 * torch.randn(K, device=DEV, generator=gen)
    if case["token_gate"]:
        s["token_gate"] = torch.sigmoid(torch.randn(N, device=DEV, generator=gen))
    if case["pre"]:
        s["w_pre"] = around_one(K)
    # a residual stream has channels far larger than the rest; a block's output less so
    s["y"] = _matrix(K, N, dtype, gen, 0.3)
    if kind == "norm":
        s["x"] = _matrix(K, N, dtype, gen, 0.8)
        return s
    s["h"] = _matrix(K, N, dtype, gen, 0.8)
    s["dh"] = _matrix(K, N, dtype, gen)
    s["du"] = _matrix(K, N, dtype, gen) if case["pre"] else None
    rstd = lambda m: torch.rsqrt(m[:, :N].float().square().mean(0) + EPS)
    s["rstd_y"] = rstd(s["y"]) if case["post"] else None
    s["rstd_h"] = rstd(s["h"]) if case["pre"] else None
    return s


def prepare(case, seed):
    kind, M, K, N, dtype = (case[k] for k in ("kind", "M", "K", "N", "dtype"))
    s = {**case, "ld": _ld(N), **_inputs(case, seed)}
    hinm = _library() if own else None
    if kind == "linear4":
        # a serving program keeps the weights in 4 bits: here the values they stand for, there the codes
        if own:
            s["W4"] = _buffers4(M, K)
            hinm.hinm_mx4_quantize(M, K, dtype, s["W"], K, hinm.MX4_ROWS, *s["W4"])
        else:
            s["W4"] = _to_4_bits(s["W"].float(), 1)
        del s["W"]
    if not own:
        return s
    f32 = lambda n, want=True: torch.empty(n, dtype=torch.float32, device=DEV) if want else None
    if kind == "weights4":
        s["W4"], s["back"] = _buffers4(M, K), torch.empty((M, K), dtype=TORCH_DTYPE[dtype], device=DEV)
    elif kind == "tokens4":
        s["X4"], s["back"] = _buffers4(N, K), torch.empty((N, K), dtype=TORCH_DTYPE[dtype], device=DEV)
    elif kind == "linear4":
        s["Y"] = _empty(M, N, dtype)
        s["workspace"] = _workspace(hinm.hinm_mx4_linear_workspace(M, K, N))
    elif kind == "linear4_grad":
        s["dX"], s["dW"] = _empty(K, N, dtype), torch.empty((M, K), dtype=torch.float32, device=DEV)
        s["WT4"], s["dYT4"], s["dY4"], s["X4"] = _buffers4(K, M), _buffers4(N, M), _buffers4(M, N), _buffers4(K, N)
    elif kind == "norm":
        s["h_out"], s["u_out"] = _empty(K, N, dtype), _empty(K, N, dtype) if case["pre"] else None
        s["rstd_y"], s["rstd_h"] = f32(N, case["post"]), f32(N, case["pre"])
        s["workspace"] = _workspace(hinm.hinm_block_norm_workspace(K, N))
    else:
        s["dx"], s["dy"] = _empty(K, N, dtype), _empty(K, N, dtype)
        s["dw_post"], s["dgate"], s["dw_pre"] = f32(K, case["post"]), f32(K, case["gate"]), f32(K, case["pre"])
        s["dtoken_gate"] = f32(N, case["token_gate"])
        s["workspace"] = _workspace(hinm.hinm_block_norm_grad_workspace(K, N))
    return s


# ---- the plain forms --------------------------------------------------------------------------------

def _to_4_bits(X, axis):
    """The values that a float32 matrix stands for after its quantisation in blocks of 32 along `axis`: the block's largest
    magnitude has its power of two brought to 4, which is the block's power of two times 4; a value over that power of two
    is rounded to the nearest of 0, .5, 1, 1.5, 2, 3, 4, 6 (ties to the even one), signs kept."""
    if axis == 0:
        return _to_4_bits(X.t(), 1).t()
    rows, n = X.shape
    pad = -n % 32
    B = (torch.nn.functional.pad(X, (0, pad)) if pad else X).reshape(rows, -1, 32)
    most = B.abs().amax(2, keepdim=True)
    power = torch.clamp(torch.frexp(most)[1] - 3, -126, 125)
    unit = ((power + 127) << 23).view(torch.float32)
    V = B / unit
    A = V.abs()
    Q = torch.where(A < 2, torch.round(A * 2) / 2, torch.where(A < 4, torch.round(A), torch.round(A / 2) * 2)).clamp(max=6)
    return (torch.copysign(Q, V) * unit).reshape(rows, n + pad)[:, :n]


def _norm_plain(s):
    N, dtype = s["N"], TORCH_DTYPE[s["dtype"]]
    x, b = s["x"][:, :N].float(), s["y"][:, :N].float()
    rstd_y = rstd_h = u = None
    if s["post"]:
        rstd_y = torch.rsqrt(b.square().mean(0) + EPS)
        b = b * rstd_y * s["w_post"][:, None]
    if s["gate"] is not None:
        b = b * s["gate"][:, None]
    if s["token_gate"] is not None:
        b = b * s["token_gate"]
    h = x * s["scale"] + b
    if s["pre"]:
        rstd_h = torch.rsqrt(h.square().mean(0) + EPS)
        u = (h * rstd_h * s["w_pre"][:, None]).to(dtype)
    return [t for t in (h.to(dtype), u, rstd_y, rstd_h) if t is not None]


def _norm_grad_of(s, as_real):
    """Gradients in the type that `as_real` converts to, by the chain rule; [dx, dy, dw_post, dgate, dtoken_gate, dw_pre]
    without those that do not exist."""
    N, K = s["N"], s["K"]
    of = lambda k: None if s[k] is None else as_real(s[k])
    cut = lambda k: as_real(s[k][:, :N])
    w_post, w_pre, gate, token_gate, rstd_y, rstd_h = (of(k) for k in ("w_post", "w_pre", "gate", "token_gate", "rstd_y", "rstd_h"))
    h, y, dh = cut("h"), cut("y"), cut("dh")
    dw_post = dgate = dtoken_gate = dw_pre = None
    if w_pre is not None:
        du, hn = cut("du"), h * rstd_h
        dw_pre = (du * hn).sum(1)
        g = du * w_pre[:, None]
        dh = dh + rstd_h * (g - hn * (g * hn).sum(0) / K)
    dx = s["scale"] * dh
    yn = y * rstd_y if w_post is not None else y
    v = yn * w_post[:, None] if w_post is not None else yn         # what the gates multiply
    channel = 1.0 if gate is None else gate[:, None]
    token = 1.0 if token_gate is None else token_gate
    if gate is not None:
        dgate = (dh * v * token).sum(1)
    if token_gate is not None:
        dtoken_gate = (dh * v * channel).sum(0)
    dv = dh * channel * token
    dy = dv
    if w_post is not None:
        dw_post = (dv * yn).sum(1)
        g = dv * w_post[:, None]
        dy = rstd_y * (g - yn * (g * yn).sum(0) / K)
    return [dx, dy, dw_post, dgate, dtoken_gate, dw_pre]


def _plain(s):
    kind, N = s["kind"], s["N"]
    dtype = TORCH_DTYPE[s["dtype"]]
    if kind == "weights4":
        return _to_4_bits(s["W"].float(), 1).to(dtype)
    if kind == "tokens4":
        return _to_4_bits(s["X"][:, :N].float(), 0).t().to(dtype)
    if kind == "linear4":
        Y = s["W4"] @ _to_4_bits(s["X"][:, :N].float(), 0)
        return (torch.relu(Y) if s["relu"] else Y).to(dtype)
    if kind == "linear4_grad":
        W, X, dY = s["W"].float(), s["X"][:, :N].float(), s["dY"][:, :N].float()
        dX = _to_4_bits(W, 0).t() @ _to_4_bits(dY, 0)
        dW = _to_4_bits(dY, 1) @ _to_4_bits(X, 1).t()
        return [dX.to(dtype), dW]
    if kind == "norm":
        return _norm_plain(s)
    dx, dy, *rest = _norm_grad_of(s, lambda t: t.float())
    return [t for t in (dx.to(dtype), dy.to(dtype), *rest) if t is not None]


# ---- one pass ---------------------------------------------------------------------------------------

def run(s):
    if not own:
        return _plain(s)
    hinm = _library()
    kind, M, K, N, dtype, ld = s["kind"], s["M"], s["K"], s["N"], s["dtype"], s["ld"]
    if kind == "weights4":
        hinm.hinm_mx4_quantize(M, K, dtype, s["W"], K, hinm.MX4_ROWS, *s["W4"])
        hinm.hinm_mx4_unpack(M, K, dtype, *s["W4"], s["back"], K)
        return s["back"]
    if kind == "tokens4":
        hinm.hinm_mx4_quantize(K, N, dtype, s["X"], ld, hinm.MX4_COLUMNS, *s["X4"])
        hinm.hinm_mx4_unpack(N, K, dtype, *s["X4"], s["back"], K)
        return s["back"]
    if kind == "linear4":
        hinm.hinm_mx4_linear(M, K, N, dtype, *s["W4"], s["X"], ld, s["Y"], ld, hinm.EPI_RELU if s["relu"] else 0,
                             *s["workspace"])
        return s["Y"][:, :N]
    if kind == "linear4_grad":
        hinm.hinm_mx4_quantize(M, K, dtype, s["W"], K, hinm.MX4_COLUMNS, *s["WT4"])
        hinm.hinm_mx4_quantize(M, N, dtype, s["dY"], ld, hinm.MX4_COLUMNS, *s["dYT4"])
        hinm.hinm_mx4_product(K, N, M, dtype, *s["WT4"], *s["dYT4"], s["dX"], ld)
        hinm.hinm_mx4_quantize(M, N, dtype, s["dY"], ld, hinm.MX4_ROWS, *s["dY4"])
        hinm.hinm_mx4_quantize(K, N, dtype, s["X"], ld, hinm.MX4_ROWS, *s["X4"])
        hinm.hinm_mx4_product(M, K, N, dtype, *s["dY4"], *s["X4"], s["dW"], K, hinm.OUT_F32)
        return [s["dX"][:, :N], s["dW"]]
    if kind == "norm":
        hinm.hinm_block_norm(K, N, dtype, s["scale"], EPS, s["x"], s["y"], s["w_post"], s["gate"], s["token_gate"], s["w_pre"],
                             s["h_out"], ld, s["u_out"], ld, s["rstd_y"], s["rstd_h"], *s["workspace"])
        out = [s["h_out"][:, :N]] + ([s["u_out"][:, :N]] if s["pre"] else [])
        return out + [t for t in (s["rstd_y"], s["rstd_h"]) if t is not None]
    hinm.hinm_block_norm_grad(K, N, dtype, s["scale"], s["h"], s["y"], s["w_post"], s["gate"], s["token_gate"], s["w_pre"],
                              s["rstd_y"], s["rstd_h"], s["dh"], s["du"], s["dx"], ld, s["dy"], ld, s["dw_post"], s["dgate"],
                              s["dtoken_gate"], s["dw_pre"], *s["workspace"])
    rest = (s["dw_post"], s["dgate"], s["dtoken_gate"], s["dw_pre"])
    return [s["dx"][:, :N], s["dy"][:, :N]] + [t for t in rest if t is not None]


# ---- from the definition, in 64 bits ------------------------------------------------------------------

def _exact_4_bits(X):
    """Values of a float64 matrix after quantisation in blocks of 32 along its rows."""
    rows, n = X.shape
    out = torch.empty_like(X)
    step = max(1, (1 << 26) // n)          # rows at a time: the comparisons below take many temporaries
    for r in range(0, rows, step):
        for_pad = torch.zeros((min(step, rows - r), -n % 32), dtype=X.dtype, device=X.device)
        B = torch.cat([X[r:r + step], for_pad], 1).reshape(-1, 32)
        A = B.abs()
        most = A.max(1, keepdim=True).values
        unit = torch.exp2(torch.floor(torch.log2(torch.where(most > 0, most, torch.ones_like(most)))) - 2)
        A = A / unit
        Q = torch.zeros_like(A)
        # a value takes the upper of two neighbours beyond their middle, and at the middle if the upper one is the even one
        for lower, upper, even in ((0, .5, 0), (.5, 1, 1), (1, 1.5, 0), (1.5, 2, 1), (2, 3, 0), (3, 4, 1), (4, 6, 0)):
            middle = (lower + upper) / 2
            Q += (upper - lower) * ((A >= middle) if even else (A > middle))
        out[r:r + step] = (torch.sign(B) * Q * unit).reshape(-1, n + -n % 32)[:, :n]
    return out


def exact(case, seed):
    kind, N = case["kind"], case["N"]
    i = _inputs(case, seed)
    if kind == "weights4":
        return _exact_4_bits(i["W"].double())
    if kind == "tokens4":
        return _exact_4_bits(i["X"][:, :N].double().t().contiguous())
    if kind == "linear4":
        X = _exact_4_bits(i["X"][:, :N].double().t().contiguous())
        Y = torch.empty((case["M"], N), dtype=torch.float64, device=DEV)
        for r in range(0, case["M"], 4096):
            Y[r:r + 4096] = torch.mm(_exact_4_bits(i["W"][r:r + 4096].double()), X.t())
        return Y.clamp(min=0) if case["relu"] else Y
    if kind == "linear4_grad":
        W, X, dY = i["W"].double(), i["X"][:, :N].double(), i["dY"][:, :N].double()
        across = lambda t: _exact_4_bits(t.t().contiguous())
        return [torch.mm(across(W), across(dY).t()), torch.mm(_exact_4_bits(dY), _exact_4_bits(X).t())]
    K = case["K"]
    get = lambda k: None if i[k] is None else i[k].double()
    w_post, gate, token_gate, w_pre = get("w_post"), get("gate"), get("token_gate"), get("w_pre")
    col = lambda t, other: torch.ones(other, 1, dtype=torch.float64, device=DEV) if t is None else t.reshape(-1, 1)
    row = lambda t: torch.ones(1, N, dtype=torch.float64, device=DEV) if t is None else t.reshape(1, -1)
    y = get("y")[:, :N]
    if kind == "norm":
        x = get("x")[:, :N]
        rstd_y = (y.pow(2).sum(0) / K + EPS).pow(-0.5) if case["post"] else None
        h = case["scale"] * x + col(gate, K) * col(w_post, K) * row(token_gate) * y * row(rstd_y)
        rstd_h = (h.pow(2).sum(0) / K + EPS).pow(-0.5) if case["pre"] else None
        u = col(w_pre, K) * h * row(rstd_h) if case["pre"] else None
        return [t for t in (h, u, rstd_y, rstd_h) if t is not None]
    # with r the given reciprocal root of a token, d/dz of w z r(z) applied to g is r w g - z r^3 <w g, z> / K
    h, d = get("h")[:, :N], get("dh")[:, :N]
    dw_pre = dw_post = dgate = dtoken = None
    if case["pre"]:
        du, r = get("du")[:, :N], get("rstd_h")
        dw_pre = torch.mv(du * h, r)
        d = d + col(w_pre, K) * du * row(r) - h * row(r.pow(3) * (col(w_pre, K) * du * h).sum(0) / K)
    r = get("rstd_y")
    along = d * y * row(r)                                    # per weight, gate and token gate of one
    if case["gate"]:
        dgate = (along * col(w_post, K) * row(token_gate)).sum(1)
    if case["token_gate"]:
        dtoken = (along * col(w_post, K) * col(gate, K)).sum(0)
    dy = d * col(gate, K) * row(token_gate)
    if case["post"]:
        dw_post = (along * col(gate, K) * row(token_gate)).sum(1)
        dy = dy * col(w_post, K)
        dy = dy * row(r) - y * row(r.pow(3) * (dy * y).sum(0) / K)
    return [t for t in (case["scale"] * d, dy, dw_post, dgate, dtoken, dw_pre) if t is not None]


# ---- what a pass cannot do without --------------------------------------------------------------------

def work(case):
    kind, M, K, N = (case[k] for k in ("kind", "M", "K", "N"))
    four = lambda n: n // 2 + n // 32            # codes and scales of n values
    if kind == "weights4":
        return {"bytes": 4 * M * K + four(M * K), "flops": 4 * M * K}
    if kind == "tokens4":
        return {"bytes": 4 * K * N + four(K * N), "flops": 4 * K * N}
    if kind == "linear4":
        return {"bytes": four(M * K) + 2 * (K + M) * N, "flops": 2 * M * K * N}
    if kind == "linear4_grad":
        return {"bytes": 2 * (M * K + K * N + M * N) + 2 * K * N + 4 * M * K, "flops": 4 * M * K * N}
    vectors = 4 * K * (case["post"] + case["gate"] + case["pre"]) + 4 * N * (case["token_gate"] + case["post"] + case["pre"])
    if kind == "norm":
        return {"bytes": 2 * K * N * (3 + case["pre"]) + vectors, "flops": K * N * (4 + 3 * case["post"] + 4 * case["pre"])}
    return {"bytes": 2 * K * N * (5 + case["pre"]) + 2 * vectors, "flops": K * N * (6 + 8 * case["post"] + 8 * case["pre"])}
