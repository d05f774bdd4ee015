"""Dense layers and layer norm together, as a program uses them: an encoder's feed-forward block forward and backward, and dense
layers in the place of compressed ones."""
import numpy as np
import pytest

from oracle import dense_oracle as orc
from tests.dense_util import DEV, HALF, TORCH, rounded

pytestmark = pytest.mark.gpu


def _block(rng, K, F, N, dtype, spare=0):
    import torch
    from paper_2407_20496_amd import binding as hb
    from paper_2407_20496_amd import block as blk
    host = {"W0": rounded(rng.normal(size=(F, K)) / np.sqrt(K), dtype), "W1": rounded(rng.normal(size=(K, F)) / np.sqrt(F), dtype)}
    for name, n in (("bias0", F), ("bias1", K), ("b", K)):
        host[name] = (0.3 * rng.normal(size=n)).astype(np.float32).astype(np.float64)
    host["w"] = (1 + 0.2 * rng.normal(size=K)).astype(np.float32).astype(np.float64)
    dev = {}
    for name, v in host.items():
        t = torch.as_tensor(v, device=DEV).to(TORCH[dtype] if name.startswith("W") else torch.float32)
        if name.startswith("W") and spare:  # rows apart
            wide = torch.full((v.shape[0], v.shape[1] + spare), float("nan"), dtype=TORCH[dtype], device=DEV)
            wide[:, :v.shape[1]] = t
            t = wide[:, :v.shape[1]]
        dev[name] = t
    layers = [blk.dense_layer(dev["W0"], dev["bias0"], hb.EPI_GELU), blk.dense_layer(dev["W1"], dev["bias1"])]
    return blk.LayerNormFeedForward(layers, N, dev["w"], dev["b"]), host


def _stream(v, dtype, ld):
    import torch
    t = torch.full((v.shape[0], ld), float("nan"), dtype=TORCH[dtype], device=DEV)
    t[:, :v.shape[1]] = torch.as_tensor(v, device=DEV).to(TORCH[dtype])
    return t


def _near(got, want, dtype, roundings, what):
    """Rounded steps in between, each off by half a step of its values at most: together, on root mean square, less than so many."""
    off = np.sqrt(((got - want) ** 2).mean() / (want ** 2).mean())
    assert off <= roundings * HALF[dtype], (what, off / HALF[dtype])


@pytest.mark.parametrize("K,F,N,dtype,spare,ld", [(96, 200, 37, "f16", 0, 40), (96, 200, 37, "bf16", 8, 43), (64, 64, 1, "bf16", 0, 1),
                                                  (256, 1024, 300, "f16", 3, 304), (250, 333, 20, "bf16", 0, 24)])
def test_a_block_forward_and_backward(K, F, N, dtype, spare, ld):
    import torch
    rng = np.random.default_rng(K + N)
    block, p = _block(rng, K, F, N, dtype, spare)
    x, dh = rounded(rng.normal(size=(K, N)) + 0.3, dtype), rounded(rng.normal(size=(K, N)), dtype)
    xd, dhd = _stream(x, dtype, ld), _stream(dh, dtype, ld)
    h = block(xd)
    dx, g = block.backward(xd, dhd)
    torch.cuda.synchronize()
    u, mean, rstd = orc.layer_norm(x, p["w"], p["b"], 1e-5)
    a, Z = orc.linear(p["W0"], u, p["bias0"], None, "gelu")
    H, _ = orc.linear(p["W1"], a, p["bias1"], x)
    _near(h[:, :N].double().cpu().numpy(), H, dtype, 3, "h")
    da, dW1, db1, _ = orc.linear_grad(p["W1"], a, None, dh)
    du, dW0, db0, _ = orc.linear_grad(p["W0"], u, Z, da, "gelu")
    DX, dw, db = orc.layer_norm_grad(x, p["w"], mean, rstd, du, dh)
    host = lambda t: t.double().cpu().numpy()
    _near(host(dx[:, :N]), DX, dtype, 6, "dx")
    for name, want in (("W0", dW0), ("W1", dW1), ("bias0", db0), ("bias1", db1), ("w", dw), ("b", db)):
        _near(host(g[name]), want, dtype, 6, name)
    # what was read is as it was, and inference gives the same
    assert torch.equal(xd[:, :N].double().cpu(), torch.as_tensor(x))
    again = h.clone()
    assert torch.equal(block(xd, train=False)[:, :N], again[:, :N])


def test_a_step_in_a_graph():
    """Captured once, replayed with other inputs, eager work in between."""
    import torch
    rng = np.random.default_rng(0)
    K, F, N = 192, 768, 200
    block, _ = _block(rng, K, F, N, "bf16")
    x, dh = (torch.randn(K, 200, device=DEV).bfloat16() for _ in range(2))

    def step():
        h = block(x)
        dx, g = block.backward(x, dh)
        return [h, dx] + list(g.values())

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for _ in range(3):
        x.copy_(torch.randn_like(x))
        dh.copy_(torch.randn_like(dh))
        want = [t.clone() for t in step()]
        for t in out:
            t.fill_(3)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


@pytest.mark.parametrize("N", [1, 20])
def test_dense_layers_in_a_block_of_norms(N):
    """FeedForward on dense layers: the same as its calls one by one."""
    import torch
    import paper_2407_20496_amd as hinm
    from paper_2407_20496_amd import block as blk
    K, F = 128, 320
    ld = blk.leading_dimension(N)
    new = lambda *s: torch.randn(*s, device=DEV).bfloat16()
    W0, W1, x, u = new(F, K), new(K, F), new(K, ld), new(K, ld)
    bias, w, w_next = (torch.randn(n, device=DEV) for n in (F, K, K))
    block = blk.FeedForward([blk.dense_layer(W0, bias, hinm.EPI_SILU), blk.dense_layer(W1)], N, w, w_next=w_next)
    a, y, h, un = new(F, ld), new(K, ld), torch.empty_like(x), torch.empty_like(u)
    scratch = torch.empty(1 << 22, dtype=torch.uint8, device=DEV)
    ws = (scratch, scratch.numel())
    hinm.hinm_linear(F, K, N, "bf16", W0, K, u, ld, bias, None, 0, None, a, ld, hinm.EPI_SILU, *ws)
    hinm.hinm_linear(K, F, N, "bf16", W1, F, a, ld, None, None, 0, None, y, ld, 0, *ws)
    hinm.hinm_block_norm(K, N, "bf16", 1.0, 1e-6, x, y, w, None, None, w_next, h, ld, un, ld, None, None, *ws)
    got_h, got_u = block(x, u)
    torch.cuda.synchronize()
    assert torch.equal(got_h[:, :N], h[:, :N]) and torch.equal(got_u[:, :N], un[:, :N])
