"""What block.py takes and refuses, on the CPU: the library's calls are recorded instead of made, and a refusal has to come
before the first of them."""
import pytest
import torch

import paper_2407_20496_amd as hinm
from paper_2407_20496_amd import block as blk

LAUNCHES = ("hinm_mx4_quantize", "hinm_mx4_product", "hinm_mx4_linear", "hinm_block_norm", "hinm_chain")
K, M, N, LD = 32, 64, 20, 24


@pytest.fixture
def calls(monkeypatch):
    made = []
    for name in LAUNCHES:
        monkeypatch.setattr(blk.hb, name, lambda *a, _n=name, **k: made.append((_n, a)))
    return made


def _layer(m, k, dtype=torch.float16, flags=0):
    return blk.Mx4Layer(m, k, dtype, *blk.mx4_form(m, k, "cpu"), flags)


def _block(dtype=torch.float16, **more):
    return blk.FeedForward([_layer(M, K, dtype), _layer(K, M, dtype)], N, torch.ones(K), w_next=torch.ones(K), device="cpu", **more)


def _new(rows=K, cols=LD, dtype=torch.float16):
    return torch.zeros((rows, cols), dtype=dtype)


BAD_ROWS = {"narrower than the tokens": lambda: _new(cols=N - 1), "too few channels": lambda: _new(rows=K - 1),
            "too many channels": lambda: _new(rows=K + 1), "another type": lambda: _new(dtype=torch.bfloat16),
            "float32": lambda: _new(dtype=torch.float32), "a vector": lambda: _new().reshape(-1),
            "columns apart": lambda: _new(cols=2 * LD)[:, ::2], "transposed": lambda: _new(rows=LD, cols=K).t(),
            "one row for all": lambda: _new(rows=1).expand(K, LD), "overlapping rows": lambda: torch.zeros(K * LD, dtype=torch.float16).as_strided((K, LD), (8, 1)),
            "another device": lambda: torch.zeros((K, LD), dtype=torch.float16, device="meta")}


@pytest.mark.parametrize("bad", BAD_ROWS.values(), ids=BAD_ROWS)
def test_a_block_refuses_other_arrays(bad, calls):
    block = _block()
    for x, u in ((bad(), _new()), (_new(), bad())):
        with pytest.raises(ValueError):
            block(x, u)
    with pytest.raises(ValueError):
        block.run_layers(bad())
    assert not calls


@pytest.mark.parametrize("cols", [N, 32])
def test_a_block_refuses_another_pitch_of_its_input(cols, calls):
    """The layers' input shares its pitch with the block's own output."""
    block = _block()
    with pytest.raises(ValueError):
        block(_new(), _new(cols=cols))
    with pytest.raises(ValueError):
        block.run_layers(_new(cols=cols))
    assert not calls


@pytest.mark.parametrize("x,pitch", [(_new(), LD), (_new(cols=N), N), (_new(cols=40), 40), (_new(cols=64)[:, :LD], 64),
                                     (_new(cols=64)[:, 8:8 + N], 64)])
def test_a_block_takes_the_pitch_of_its_stream(x, pitch, calls):
    _block()(x, _new())
    name, args = calls[-1]
    assert name == "hinm_block_norm" and args[5] is x and args[11] is x and args[12] == pitch and args[14] == LD


def test_a_wider_view_is_as_good_as_a_buffer_of_the_blocks_pitch(calls):
    u = _new(cols=LD)[:, :N]
    assert _block().run_layers(u) is not None and calls[0][0] == "hinm_mx4_linear" and calls[0][1][7] == LD


BAD_VECTORS = {"float64": torch.ones(K, dtype=torch.float64), "bfloat16": torch.ones(K, dtype=torch.bfloat16), "short": torch.ones(N - 1),
               "apart": torch.ones(2 * K)[::2], "one for all": torch.ones(1).expand(K), "another device": torch.ones(K, device="meta")}


@pytest.mark.parametrize("bad", BAD_VECTORS.values(), ids=BAD_VECTORS)
def test_a_block_refuses_other_factors(bad, calls):
    layers = [_layer(M, K), _layer(K, M)]
    for w_post, gate, w_next in ((bad, None, None), (None, bad, None), (None, None, bad)):
        with pytest.raises(ValueError):
            blk.FeedForward(layers, N, w_post, gate, w_next, device="cpu")
    with pytest.raises(ValueError):
        blk.block_input(_new(), bad, N)
    with pytest.raises(ValueError):
        _block()(_new(), _new(), token_gate=bad)
    assert not calls


def test_a_block_takes_factors_of_any_shape_and_room_for_more_tokens(calls):
    block = blk.FeedForward([_layer(M, K), _layer(K, M)], N, torch.ones(K, 1), torch.ones(1, K), torch.ones(K), device="cpu")
    block(_new(), _new(), token_gate=torch.ones(N + 5))
    assert calls[-1][0] == "hinm_block_norm"


@pytest.mark.parametrize("x,pitch", [(_new(cols=1), 1), (_new(cols=1).reshape(-1), 1), (_new()[:, 3:4], LD), (_new()[:, 3], LD)])
def test_one_token_may_be_a_vector(x, pitch, calls):
    block = blk.FeedForward([_layer(M, K), _layer(K, M)], 1, torch.ones(K), w_next=torch.ones(K), device="cpu")
    u = _new(cols=1).reshape(x.shape)
    assert block(x, u)[1] is u and calls[-1][1][12] == pitch and calls[-1][1][14] == 1
    with pytest.raises(ValueError):
        block(x[1:], u)


def test_a_blocks_layers_share_their_type_and_device():
    with pytest.raises(ValueError):
        blk.FeedForward([_layer(M, K), _layer(K, M, torch.bfloat16)], N, None, device="cpu")
    with pytest.raises(ValueError):
        blk.FeedForward([_layer(M, K), _layer(K, M)], N, None, device="meta")
    assert blk.FeedForward([_layer(M, K, "f16"), _layer(K, M, hinm.F16)], N, None, device="cpu").y.dtype == torch.float16


@pytest.mark.parametrize("bad", [k for k in BAD_ROWS if "channels" not in k and k not in ("another type", "another device")])
def test_a_blocks_input_refuses_other_arrays(bad, calls):
    x = BAD_ROWS[bad]()
    with pytest.raises(ValueError):
        blk.block_input(x, torch.ones(K), N)
    assert not calls


@pytest.mark.parametrize("x,pitch", [(_new(), LD), (_new(cols=N), N), (_new(cols=64)[:, :LD], 64), (_new(cols=1), 1)])
def test_a_blocks_input_has_the_shape_of_its_stream(x, pitch, calls):
    u = blk.block_input(x, torch.ones(K), min(N, x.shape[1]))
    args = calls[-1][1]
    assert u.shape == x.shape and u.is_contiguous() and args[5] is x and args[12] == pitch and args[14] == x.shape[1]


def _strided(rows, cols, *strides):
    return torch.zeros(rows * cols + 64 * sum(strides), dtype=torch.bfloat16).as_strided((rows, cols), strides)


@pytest.mark.parametrize("W", [torch.zeros(1, K, dtype=torch.bfloat16).expand(M, K), _strided(M, K, 8, 1), _strided(M, K, K - 1, 1),
                               _strided(M, K, 1, M), _strided(M, K, 2 * K, 2), torch.zeros(M * K, dtype=torch.bfloat16),
                               torch.zeros(M, K, 1, dtype=torch.bfloat16), torch.zeros(M, K)],
                         ids=["one row for all", "overlapping", "overlapping by one", "transposed", "columns apart", "a vector", "a cube", "float32"])
def test_a_layer_refuses_weights_that_do_not_lie_row_by_row(W, calls):
    with pytest.raises(ValueError):
        blk.mx4_layer(W)
    assert not calls


@pytest.mark.parametrize("W,pitch", [(_strided(M, K, K, 1), K), (_strided(M, K, K + 5, 1), K + 5), (_strided(1, K, 0, 1), K), (_strided(1, K, 7, 1), K),
                                     (_strided(M, 1, 3, 5), 3)])
def test_a_layer_takes_the_pitch_of_its_weights(W, pitch, calls):
    layer = blk.mx4_layer(W)
    assert (layer.M, layer.K) == W.shape and calls[0][1][3] is W and calls[0][1][4] == pitch


BF16 = torch.bfloat16
GOOD = {"W": lambda: _new(M, K, BF16), "X": lambda: _new(K, LD, BF16), "dY": lambda: _new(M, LD, BF16)}
BAD = {"W": {"float32": lambda: _new(M, K, torch.float32), "another type": lambda: _new(M, K), "transposed": lambda: _new(K, M, BF16).t(),
             "one row for all": lambda: _new(1, K, BF16).expand(M, K), "columns apart": lambda: _new(M, 2 * K, BF16)[:, ::2],
             "a vector": lambda: _new(M, K, BF16).reshape(-1), "another device": lambda: _new(M, K, BF16).to("meta")},
       "X": {"another type": lambda: _new(K, LD), "too few channels": lambda: _new(K - 1, LD, BF16), "too many channels": lambda: _new(M, LD, BF16),
             "narrower than the tokens": lambda: _new(K, N - 1, BF16), "transposed": lambda: _new(LD, K, BF16).t(),
             "overlapping": lambda: _strided(K, LD, 8, 1), "another device": lambda: _new(K, LD, BF16).to("meta")},
       "dY": {"another type": lambda: _new(M, LD), "too few rows": lambda: _new(K, LD, BF16), "too many rows": lambda: _new(M + 1, LD, BF16),
              "narrower than the tokens": lambda: _new(M, N - 1, BF16), "columns apart": lambda: _new(M, 2 * LD, BF16)[:, ::2],
              "another device": lambda: _new(M, LD, BF16).to("meta")}}


@pytest.mark.parametrize("which,what", [(k, w) for k, v in BAD.items() for w in v])
def test_a_layers_gradients_refuse_other_arrays(which, what, calls):
    given = {k: v() for k, v in GOOD.items()}
    given[which] = BAD[which][what]()
    with pytest.raises(ValueError):
        blk.mx4_linear_grad(**given, tokens=N)
    assert not calls


def test_a_layers_gradients_refuse_as_many_tokens_as_there_are_in_one_array_only(calls):
    with pytest.raises(ValueError):
        blk.mx4_linear_grad(GOOD["W"](), _new(K, 2 * LD, BF16), GOOD["dY"]())
    assert not calls


@pytest.mark.parametrize("cols_w,cols_x,cols_dy", [(K, LD, LD), (K + 3, LD, LD), (K, 40, LD), (K, LD, 64), (2 * K, N, 41)])
def test_a_layers_gradients_take_the_pitch_of_each_array(cols_w, cols_x, cols_dy, calls):
    W, X, dY = _new(M, cols_w, BF16)[:, :K], _new(K, cols_x, BF16)[:, :N], _new(M, cols_dy, BF16)[:, :N]
    dX, dW = blk.mx4_linear_grad(W, X, dY)
    assert dX.shape == X.shape and dX.is_contiguous() and dW.shape == W.shape
    quantised = {(a[3].data_ptr(), a[5]): a[:5] for n, a in calls if n == "hinm_mx4_quantize"}
    assert quantised[W.data_ptr(), hinm.MX4_COLUMNS] == (M, K, BF16, W, cols_w)
    assert quantised[X.data_ptr(), hinm.MX4_ROWS] == (K, N, BF16, X, cols_x)
    assert quantised[dY.data_ptr(), hinm.MX4_COLUMNS] == quantised[dY.data_ptr(), hinm.MX4_ROWS] == (M, N, BF16, dY, cols_dy)
    products = [(a[:3], a[8], a[9]) for n, a in calls if n == "hinm_mx4_product"]
    assert products == [((K, N, M), dX, N), ((M, K, N), dW, K)]


@pytest.mark.parametrize("which", ["codes", "scales"])
def test_a_block_refuses_layers_with_less_memory_than_their_form_has(which):
    for cut in (lambda t: t[:-1], lambda t: t.view(torch.int16), lambda t: t.repeat(2)[::2]):
        short = _layer(M, K)
        setattr(short, which, cut(getattr(short, which)))
        with pytest.raises(ValueError):
            blk.FeedForward([short, _layer(K, M)], N, None, device="cpu")
