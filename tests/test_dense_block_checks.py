"""What block.py takes and refuses of dense layers, on the CPU: the library's calls are recorded instead of made, and a refusal has
to come before the first of them."""
import pytest
import torch

from paper_2407_20496_amd import binding as hb
from paper_2407_20496_amd import block as blk

K, F, N, LD = 32, 64, 20, 24
LAUNCHES = ("hinm_linear", "hinm_linear_grad", "hinm_layer_norm", "hinm_layer_norm_grad", "hinm_block_norm")


@pytest.fixture
def calls(monkeypatch):
    made = []
    for name in LAUNCHES:
        monkeypatch.setattr(blk.hb, name, lambda *a, _n=name, **k: made.append((_n, a)))
    return made


def _new(rows=K, cols=LD, dtype=torch.float16):
    return torch.zeros((rows, cols), dtype=dtype)


def _layers():
    return [blk.dense_layer(_new(F, K), torch.zeros(F), hb.EPI_GELU), blk.dense_layer(_new(K, F), torch.zeros(K))]


def _block(**more):
    return blk.LayerNormFeedForward(_layers(), N, torch.ones(K), torch.zeros(K), device="cpu", **more)


@pytest.mark.parametrize("make", [
    lambda: blk.dense_layer(torch.zeros(4, 4)), lambda: blk.dense_layer(_new(4, 4).t()[:, ::2]), lambda: blk.dense_layer(_new(1, 8).expand(4, 8)),
    lambda: blk.dense_layer(_new(4, 8), torch.zeros(3)), lambda: blk.dense_layer(_new(4, 8), torch.zeros(4, dtype=torch.float64)),
    lambda: blk.dense_layer(_new(4, 8), None, hb.EPI_GELU | hb.EPI_SILU), lambda: blk.dense_layer(_new(4, 8), None, hb.OUT_F32)])
def test_layers_refused(make):
    with pytest.raises(ValueError):
        make()


@pytest.mark.parametrize("layers", [
    lambda: [], lambda: _layers()[:1], lambda: _layers()[::-1] + _layers()[:1], lambda: [_layers()[0], blk.dense_layer(_new(K, F, torch.bfloat16))],
    lambda: [_layers()[0], blk.dense_layer(_new(K, F), None, hb.EPI_RELU)], lambda: [blk.Mx4Layer(K, K, torch.float16, *blk.mx4_form(K, K, "cpu"))],
    lambda: [_layers()[0], blk.DenseLayer(K, F, torch.float16, _new(K, F - 1))], lambda: [_layers()[0], blk.dense_layer(_new(K, F).to("meta"))]])
def test_blocks_refused(layers):
    with pytest.raises(ValueError):
        blk.LayerNormFeedForward(layers(), N, device="cpu")


def test_norm_weights_refused():
    for bad in (torch.ones(K - 1), torch.ones(K, dtype=torch.float16), torch.ones(2 * K)[::2]):
        with pytest.raises(ValueError):
            blk.LayerNormFeedForward(_layers(), N, bad, device="cpu")
        with pytest.raises(ValueError):
            blk.LayerNormFeedForward(_layers(), N, None, bad, device="cpu")


BAD = {"narrow": lambda: _new(cols=N - 1), "few channels": lambda: _new(rows=K - 1), "another type": lambda: _new(dtype=torch.bfloat16),
       "columns apart": lambda: _new(cols=2 * LD)[:, ::2], "one row for all": lambda: _new(rows=1).expand(K, LD),
       "another device": lambda: _new().to("meta")}


@pytest.mark.parametrize("bad", BAD.values(), ids=BAD)
def test_arrays_refused(bad, calls):
    block = _block()
    with pytest.raises(ValueError):
        block(bad())
    for x, dh in ((bad(), _new()), (_new(), bad())):
        with pytest.raises(ValueError):
            block.backward(x, dh)
    assert not calls


def test_another_pitch_of_the_gradient_is_refused(calls):
    with pytest.raises(ValueError):
        _block().backward(_new(), _new(cols=32))
    assert not calls


def test_calls_of_a_step(calls):
    x, dh = _new(cols=40)[:, :N], _new(cols=40)
    block = _block()
    block(x)
    block.backward(x, dh)
    assert [c[0] for c in calls] == ["hinm_layer_norm", "hinm_linear", "hinm_linear", "hinm_linear_grad", "hinm_linear_grad",
                                     "hinm_layer_norm_grad"]
    last = calls[2][1]
    assert last[9] is x and last[10] == 40 and last[12] is block.h and last[13] == LD
    assert calls[5][1][4] == 40 and calls[5][1][11].shape[1] == 40


def test_rows_of_weights_apart(calls):
    """dW is contiguous: asked for in a call of its own where W is not."""
    W = _new(F, K + 8)[:, :K]
    block = blk.LayerNormFeedForward([blk.dense_layer(W), blk.dense_layer(_new(K, F))], N, device="cpu")
    block.backward(_new(), _new())
    pitches = [(c[1][5], c[1][11] is not None, c[1][12] is not None) for c in calls if c[0] == "hinm_linear_grad"]
    assert pitches == [(F, True, True), (K + 8, True, False), (K, False, True)]


def test_dense_layers_are_not_mixed():
    other = blk.Mx4Layer(K, F, torch.float16, *blk.mx4_form(K, F, "cpu"))
    with pytest.raises(ValueError):
        blk.FeedForward([_layers()[0], other], N, torch.ones(K), device="cpu")


def test_no_backward_pass_behind_a_call_that_kept_nothing(calls):
    """Z would be an earlier step's."""
    block = _block()
    block(_new())
    block(_new(), train=False)
    made = len(calls)
    with pytest.raises(ValueError):
        block.backward(_new(), _new())
    assert len(calls) == made
    block(_new())
    block.backward(_new(), _new())
