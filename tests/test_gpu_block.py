"""The feed-forward block of block.py: every stage against the binary64 oracle on what the stage before it left, with 4-bit
layers and with HiNM layers, two blocks in a row."""
import numpy as np
import pytest

import hinm_synth as synth
from oracle import block_oracle as orc
from oracle import hinm_oracle as sparse

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
EPS = 1e-6
HALF_STEP = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}   # of 11 and 8 significant bits


def _wide(t, N):
    return t[:, :N].float().cpu().numpy().astype(np.float64)


def _close(got, want, size, dtype, roundings):
    """Half a step of the storage type, and fp32 roundings of 2^-24 of the magnitudes that meet."""
    tiny = 2.0 ** -25 if dtype == "f16" else 0
    assert (np.abs(got - want) <= HALF_STEP[dtype] * np.abs(want) + roundings * 2.0 ** -24 * size + tiny).all()


def _mx4(hinm, blk, K, M, dtype, kind, rng, torch):
    dense = [torch.from_numpy(rng.standard_normal(s).astype(np.float32) * 0.05).to(kind).to(DEV) for s in ((M, K), (K, M))]
    layers = [blk.mx4_layer(dense[0], hinm.EPI_RELU), blk.mx4_layer(dense[1])]
    values = [orc.values(*orc.quantize_rows(w.float().cpu().numpy().astype(np.float64)), w.shape[1]) for w in dense]

    def apply(i, X):
        Q = orc.values(*orc.quantize_rows(np.ascontiguousarray(X.T)), X.shape[0])
        return orc.product(values[i], Q, relu=i == 0)
    return layers, apply


def _sparse(hinm, K, M, dtype, rng):
    from tests import gpu_util as gu
    layers, weights = [], []
    for i, (m, k) in enumerate(((M, K), (K, M))):
        W = synth.to_bits(rng.standard_normal((m, k)).astype(np.float32) * 0.05, dtype)
        p = gu.gpu_pack(W, dtype, 32, k // 2)
        pr = gu.gpu_prepare(p, np.arange(k, dtype=np.int32), np.arange(m, dtype=np.int32))
        layers.append(hinm.Layer(m, k, 32, k // 2, dtype, p.vals, p.nm_idx, p.vec_idx, None, None, hinm.EPI_RELU if i == 0 else 0,
                                 pr.buf))
        weights.append(sparse.decode(sparse.unpack(*p.host(), m, k, 32), dtype).astype(np.float64))

    def apply(i, X):
        Y, size = weights[i] @ X, np.abs(weights[i]) @ np.abs(X)
        return (np.maximum(Y, 0) if i == 0 else Y), size
    return layers, apply


@pytest.mark.parametrize("form", ["mx4", "sparse"])
@pytest.mark.parametrize("N,dtype", [(1, "bf16"), (20, "f16"), (70, "bf16")])
def test_two_blocks(form, N, dtype):
    import torch
    import paper_2407_20496_amd as hinm
    from paper_2407_20496_amd import block as blk
    K, M = 192, 320
    kind = {"f16": torch.float16, "bf16": torch.bfloat16}[dtype]
    rng = np.random.default_rng(N)
    vec = lambda n: torch.from_numpy((1 + 0.2 * rng.standard_normal(n)).astype(np.float32)).to(DEV)
    f64 = lambda t: t.cpu().numpy().astype(np.float64)
    x = torch.zeros((K, blk.leading_dimension(N)), dtype=kind, device=DEV)
    x[:, :N] = torch.from_numpy(rng.standard_normal((K, N)).astype(np.float32)).to(kind).to(DEV)
    w_pre, token_gate = vec(K), torch.from_numpy(rng.random(N).astype(np.float32)).to(DEV)
    u = blk.block_input(x, w_pre, N, EPS)
    r = orc.block_norm(_wide(x, N), None, None, None, None, f64(w_pre), 1.0, np.float32(EPS))
    _close(_wide(u, N), r["u"], np.abs(r["u"]), dtype, K)
    for last in (False, True):
        layers, apply = _mx4(hinm, blk, K, M, dtype, kind, rng, torch) if form == "mx4" else _sparse(hinm, K, M, dtype, rng)
        w_post, gate, w_next = vec(K), vec(K), None if last else vec(K)
        block = blk.FeedForward(layers, N, w_post, gate, w_next, residual_scale=0.5, eps=EPS, device=DEV)
        y = _wide(block.run_layers(u), N)
        if form == "mx4":
            first, size = apply(0, _wide(u, N))
            _close(_wide(block.between[0], N), first, size, dtype, K)
            want, size = apply(1, _wide(block.between[0], N))
            _close(y, want, size, dtype, M)
        else:  # the chain keeps its intermediate to itself: its rounding reaches y through the second layer
            first, of_first = apply(0, _wide(u, N))
            slack = HALF_STEP[dtype] * np.abs(first) + (K * 2.0 ** -24) * of_first + (2.0 ** -25 if dtype == "f16" else 0)
            want, size = apply(1, first)
            assert (np.abs(y - want) <= HALF_STEP[dtype] * np.abs(want) * 1.01 + apply(1, slack)[1] * 1.01 + M * 2.0 ** -24 * size
                    + (2.0 ** -25 if dtype == "f16" else 0)).all()
        before = _wide(x, N)
        kept = u.clone()
        x2, u2 = block(x, u, token_gate)
        assert x2 is x and u2 is u and np.array_equal(_wide(block.y, N), y)
        r = orc.block_norm(before, y, f64(w_post), f64(gate), f64(token_gate), None if last else f64(w_next), 0.5, np.float32(EPS))
        _close(_wide(x, N), r["h"], r["size"], dtype, K)
        if last:
            assert torch.equal(u, kept)
        else:
            of_h = np.sqrt((r["size"] ** 2).mean(axis=0)) * r["rstd_h"]
            _close(_wide(u, N), r["u"], np.abs(f64(w_next))[:, None] * r["rstd_h"] * r["size"] * (1 + of_h), dtype, K)


def test_gradients_of_a_4_bit_layer():
    """Straight-through: the gradients are those of the products on quantised operands."""
    import torch
    from paper_2407_20496_amd import block as blk
    M, K, N, ld = 96, 200, 50, 56
    rng = np.random.default_rng(5)
    draw = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).to(torch.bfloat16).to(DEV)
    W, X, dY = draw(M, K), draw(K, ld), draw(M, ld)
    dX, dW = blk.mx4_linear_grad(W, X, dY, N)
    q = lambda a: orc.values(*orc.quantize_rows(np.ascontiguousarray(a)), a.shape[1])
    w, x, g = W.float().cpu().numpy().astype(np.float64), _wide(X, N), _wide(dY, N)
    want, size = orc.product(q(w.T), q(g.T))
    _close(_wide(dX, N), want, size, "bf16", M)
    want, size = orc.product(q(g), q(x))
    assert (np.abs(dW.cpu().numpy() - want) <= N * 2.0 ** -24 * size).all()
    only = blk.mx4_linear_grad(W, X, dY, N, want_weights=False)
    assert only[1] is None and torch.equal(only[0][:, :N], dX[:, :N])


def test_what_a_block_refuses():
    import torch
    import paper_2407_20496_amd as hinm
    from paper_2407_20496_amd import block as blk
    W = torch.zeros((64, 32), dtype=torch.float16, device=DEV)
    up, down = blk.mx4_layer(W), blk.mx4_layer(W.t().contiguous())
    ones = torch.ones(32, device=DEV)
    with pytest.raises(ValueError):
        blk.FeedForward([up], 4, ones)
    with pytest.raises(ValueError):
        blk.FeedForward([], 4, ones)
    with pytest.raises(ValueError):
        blk.FeedForward([up, hinm.Layer(32, 64, 32, 32, "f16", None, None, None)], 4, ones)
    with pytest.raises(ValueError):
        blk.mx4_layer(W.t())
    assert blk.FeedForward([up, down], 4, ones).y.shape == (32, 8)
