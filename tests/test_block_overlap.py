"""Arrays that share memory with a block's own buffers, on the CPU: the library's calls are recorded instead of made."""
import pytest
import torch

import paper_2407_20496_amd as hinm
from paper_2407_20496_amd import block as blk

K, F, N, LD = 32, 64, 20, 24
LAUNCHES = ("hinm_linear", "hinm_linear_grad", "hinm_layer_norm", "hinm_layer_norm_grad", "hinm_block_norm", "hinm_mx4_linear")


@pytest.fixture
def calls(monkeypatch):
    made = []
    for name in LAUNCHES:
        monkeypatch.setattr(blk.hb, name, lambda *a, _n=name, **k: made.append(_n))
    return made


def _new(rows=K, cols=LD):
    return torch.zeros((rows, cols), dtype=torch.float16)


def _dense(m, k):
    return blk.dense_layer(_new(m, k))


def _mx4(m, k):
    return blk.Mx4Layer(m, k, torch.float16, *blk.mx4_form(m, k, "cpu"))


def _block():
    return blk.LayerNormFeedForward([_dense(F, K), _dense(K, F)], N, device="cpu")


def test_a_blocks_result_may_be_its_next_input(calls):
    """In place: h takes the place of the x that a backward pass would read."""
    block = _block()
    for again in (lambda h: h, lambda h: h[:, :N], lambda h: h.view(K, LD)):
        block(again(block(_new())))
        made = len(calls)
        with pytest.raises(ValueError):
            block.backward(block.h, _new())
        with pytest.raises(ValueError):
            block.backward(_new(), _new())
        assert len(calls) == made
    block(_new())
    block.backward(_new(), _new())


def test_a_backward_pass_of_what_the_call_overwrote_is_refused(calls):
    """x = h, which holds the call's result by now; as a gradient h is as good as another array."""
    block = _block()
    block(_new())
    made = len(calls)
    with pytest.raises(ValueError):
        block.backward(block.h, _new())
    assert len(calls) == made
    block.backward(_new(), block.h)


def _shifted(t):
    """Rows of the same pitch, over the same memory but for a few values."""
    return t.reshape(-1)[4:].as_strided((K, N), (LD, 1))


def _halved(t):
    """Rows of another pitch over the same memory."""
    return t.reshape(-1).as_strided((K, N), (N, 1))


@pytest.mark.parametrize("other", [_shifted, _halved])
def test_another_part_of_a_blocks_result_is_no_input(other, calls):
    block = _block()
    block(_new())
    made = len(calls)
    with pytest.raises(ValueError):
        block(other(block.h))
    assert len(calls) == made
    block.backward(_new(), _new())  # the step before it is as it was


def test_a_blocks_gradient_may_come_back(calls):
    """dx may be dh, in place; what lies over it in another way, and an x in its place, may not."""
    block = _block()
    block(_new())
    dx, _ = block.backward(_new(), _new())
    assert block.backward(_new(), dx)[0] is dx
    made = len(calls)
    for x, dh in ((_new(), _shifted(dx)), (dx, _new()), (_shifted(dx), _new())):
        with pytest.raises(ValueError):
            block.backward(x, dh)
    assert len(calls) == made


@pytest.mark.parametrize("layer,call", [(_dense, "hinm_linear"), (_mx4, "hinm_mx4_linear")])
def test_one_layer_does_not_read_what_it_writes(layer, call, calls):
    one = blk.FeedForward([layer(K, K)], N, None, device="cpu")
    y = one.run_layers(_new())
    made = len(calls)
    for u in (y, y[:, :N], _shifted(y)):
        with pytest.raises(ValueError):
            one.run_layers(u)
        with pytest.raises(ValueError):
            one(_new(), u)
    assert len(calls) == made
    two = blk.FeedForward([layer(F, K), layer(K, F)], N, None, device="cpu")  # what lies between them is apart
    assert two.run_layers(two.run_layers(_new())) is two.y and calls[made:] == 4 * [call]
    with pytest.raises(ValueError):
        two.run_layers(_shifted(two.y))


def test_one_channel(calls):
    """One row has no pitch."""
    block = blk.LayerNormFeedForward([_dense(F, 1), _dense(1, F)], N, device="cpu")
    block(block(_new(1))[:, :N])
    with pytest.raises(ValueError):
        block.backward(_new(1), _new(1))


def test_neighbours_in_one_allocation_do_not_overlap():
    """What lies right ahead of a buffer and right behind it is another array; one value more is not."""
    whole = torch.zeros(3 * K * LD, dtype=torch.float16)
    ahead, own, behind = (t.view(K, LD) for t in whole.split(K * LD))
    place = blk._place(own)
    assert not blk._is_own(ahead, LD, "x", LD, place) and not blk._is_own(behind, LD, "x", N, place) and blk._is_own(own, LD, "x", N, place)
    for first in (K * LD - (LD - N) + 1, 2 * K * LD - 1):
        with pytest.raises(ValueError):
            blk._is_own(whole[first:].as_strided((K, N), (LD, 1)) if first < K * LD else whole[first:].view(1, -1), LD, "x", N, place)
    assert not blk._is_own(whole[LD - N:].as_strided((K, N), (LD, 1)), LD, "x", N, place)  # its last row ends where the buffer begins
