"""A feed-forward block on residual streams of other pitches: as wide as its tokens, wider, and columns of a larger matrix."""
import numpy as np
import pytest

from oracle import block_oracle as orc
from tests.test_gpu_block import DEV, EPS, _close, _mx4, _sparse, _wide

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("form", ["mx4", "sparse"])
@pytest.mark.parametrize("K,M,N", [(96, 64, 20), (1056, 96, 70)])
@pytest.mark.parametrize("width,first", [(0, 0), (128, 0), (131, 3)])
def test_a_stream_of_another_pitch(form, K, M, N, width, first):
    import torch
    import paper_2407_20496_amd as hinm
    from paper_2407_20496_amd import block as blk
    rng = np.random.default_rng(K + N)
    draw = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).to(torch.bfloat16).to(DEV)
    vec = lambda n: torch.from_numpy((1 + 0.2 * rng.standard_normal(n)).astype(np.float32)).to(DEV)
    f64 = lambda t: t.cpu().numpy().astype(np.float64)
    buffer = draw(K, width or N)
    x, u = buffer[:, first:first + N], draw(K, blk.leading_dimension(N))
    layers, _ = _mx4(hinm, blk, K, M, "bf16", torch.bfloat16, rng, torch) if form == "mx4" else _sparse(hinm, K, M, "bf16", rng)
    w_post, w_next = vec(K), vec(K)
    block = blk.FeedForward(layers, N, w_post, None, w_next, eps=EPS, device=DEV)
    before, around = _wide(x, N), buffer.clone()
    y = _wide(block.run_layers(u), N)
    block(x, u)
    r = orc.block_norm(before, y, f64(w_post), None, None, f64(w_next), 1.0, np.float32(EPS))
    _close(_wide(x, N), r["h"], r["size"], "bf16", K)
    of_h = np.sqrt((r["size"] ** 2).mean(axis=0)) * r["rstd_h"]
    _close(_wide(u, N), r["u"], np.abs(f64(w_next))[:, None] * r["rstd_h"] * r["size"] * (1 + of_h), "bf16", K)
    for at in (slice(0, first), slice(first + N, None)):
        assert torch.equal(buffer[:, at], around[:, at])
    t = blk.block_input(x, w_next, N, EPS)
    want = orc.block_norm(_wide(x, N), None, None, None, None, f64(w_next), 1.0, np.float32(EPS))["u"]
    assert t.shape == x.shape
    _close(_wide(t, N), want, np.abs(want), "bf16", K)


def test_gradients_of_a_layer_from_slices_of_larger_arrays():
    """The same values at other pitches: the same gradients, bit for bit."""
    import torch
    from paper_2407_20496_amd import block as blk
    M, K, N = 130, 200, 51
    rng = np.random.default_rng(6)
    draw = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).to(torch.bfloat16).to(DEV)
    W, X, dY = draw(M, K + 9)[:, 3:3 + K], draw(K, 64)[:, :N], draw(M, N + 2)[:, 1:1 + N]
    got = blk.mx4_linear_grad(W, X, dY)
    want = blk.mx4_linear_grad(W.contiguous(), X.contiguous(), dY.contiguous())
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    layer, same = blk.mx4_layer(W), blk.mx4_layer(W.contiguous())
    held = torch.arange(32 * ((M + 31) // 32), device=DEV).reshape(-1, 32) < M          # rows that exist
    codes = lambda l: l.codes.reshape(-1, held.shape[0], 8, 32, 16).transpose(2, 3)[:, held]
    assert torch.equal(codes(layer), codes(same))
