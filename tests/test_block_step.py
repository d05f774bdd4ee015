"""Which step a backward pass of LayerNormFeedForward belongs to, on the CPU: the library's calls are recorded instead of made."""
import pytest
import torch

import paper_2407_20496_amd as hinm
from paper_2407_20496_amd import block as blk

K, F, N, LD = 32, 64, 20, 24
LAUNCHES = ("hinm_linear", "hinm_linear_grad", "hinm_layer_norm", "hinm_layer_norm_grad")
FORWARD = ["hinm_layer_norm", "hinm_linear", "hinm_linear"]
BACKWARD = ["hinm_linear_grad", "hinm_linear_grad", "hinm_layer_norm_grad"]


class Calls(list):
    fails = None  # the name of a call that is to raise

    def made(self):
        names = [n for n, _ in self]
        self.clear()
        return names


@pytest.fixture
def calls(monkeypatch):
    made = Calls()

    def record(name, args):
        made.append((name, args))
        if made.fails == name:
            raise hinm.HinmError(6, name)

    for name in LAUNCHES:
        monkeypatch.setattr(blk.hb, name, lambda *a, _n=name, **k: record(_n, a))
    return made


def _new(rows=K, cols=LD):
    return torch.zeros((rows, cols), dtype=torch.float16)


def _block():
    layers = [blk.dense_layer(_new(F, K), torch.zeros(F), hinm.EPI_GELU), blk.dense_layer(_new(K, F), torch.zeros(K))]
    return blk.LayerNormFeedForward(layers, N, torch.ones(K), torch.zeros(K), device="cpu")


def test_a_backward_pass_ahead_of_any_call_makes_the_call(calls):
    """The block's buffers hold nothing yet: it computes from x what it needs, Z among it, and not from what memory held."""
    block, x, dh = _block(), _new(), _new()
    block.backward(x, dh)
    assert calls[0][1][4] is x and calls[1][1][11] is block.Z[0]
    assert calls.made() == FORWARD + BACKWARD
    block.backward(x, dh)
    assert calls.made() == BACKWARD


def test_refused_arrays_make_no_call(calls):
    block = _block()
    for x, dh in ((_new(K - 1), _new()), (_new(), _new(K - 1)), (_new(), _new(cols=32))):
        with pytest.raises(ValueError):
            block.backward(x, dh)
    assert not calls


@pytest.mark.parametrize("fails", ["hinm_layer_norm", "hinm_linear"])
@pytest.mark.parametrize("before", [0, 1])
def test_no_backward_pass_behind_a_call_that_failed(calls, fails, before):
    """Part of what a step keeps would be an earlier one's, or nothing at all."""
    block = _block()
    for _ in range(before):
        block(_new())
    calls.fails = fails
    with pytest.raises(hinm.HinmError):
        block(_new())
    calls.fails = None
    calls.made()
    with pytest.raises(ValueError):
        block.backward(_new(), _new())
    assert not calls
    block(_new())
    block.backward(_new(), _new())
    assert calls.made() == FORWARD + BACKWARD


def test_no_backward_pass_behind_refused_activations(calls):
    """A refused array leaves the step before it as it was."""
    block = _block()
    block(_new())
    with pytest.raises(ValueError):
        block(_new(K - 1))
    calls.made()
    block.backward(_new(), _new())
    assert calls.made() == BACKWARD


@pytest.mark.gpu
@pytest.mark.parametrize("K,F,N", [(96, 200, 37), (64, 64, 1)])
def test_a_backward_pass_ahead_of_any_call_is_that_of_a_step(K, F, N):
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(K)
    new = lambda *s: torch.randn(*s, device="cuda:0", generator=gen)
    ld = blk.leading_dimension(N)
    layers = [blk.dense_layer(new(F, K).half(), new(F), hinm.EPI_GELU), blk.dense_layer(new(K, F).half(), new(K))]
    x, dh, w, b = new(K, ld).half(), new(K, ld).half(), new(K), new(K)
    first, second = (blk.LayerNormFeedForward(layers, N, w, b) for _ in range(2))
    for block in (first, second):
        for t in [block.u, block.h, block.mean, block.rstd, *block.out] + [z for z in block.Z if z is not None]:
            t.fill_(float("nan"))
    second(x)
    (dx, got), (dx2, want) = first.backward(x, dh), second.backward(x, dh)
    assert torch.isfinite(dx[:, :N]).all() and torch.equal(dx[:, :N], dx2[:, :N]) and got.keys() == want.keys()
    assert all(torch.isfinite(got[k]).all() and torch.equal(got[k], want[k]) for k in want)
