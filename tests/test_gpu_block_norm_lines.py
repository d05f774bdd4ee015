"""Norms and gradients over matrices whose rows are whole cache lines, by several strips of tokens: the order of the list of strips,
stores around the caches, strips added by a launch of their own; full strips of 64 and cut ones, channels that fill no patch."""
import pytest

from tests.test_gpu_block_norm import _backward, _forward

pytestmark = pytest.mark.gpu

ALL = dict(post=1, gate=1, token=1, pre=1, block=1)
SIZES = [(1100, 64, 64), (1100, 128, 128), (4100, 192, 192), (1100, 190, 192), (1100, 130, 256), (1059, 65, 128), (2200, 1000, 1024), (1100, 4096, 4096),
         (11008, 321, 384)]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("K,N,ld", SIZES)
def test_forward(K, N, ld, in_place, dtype):
    _forward(K, N, dtype, ALL, ld, ld, 0, K + N, in_place=in_place)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("K,N,ld", SIZES)
def test_backward(K, N, ld, in_place, dtype):
    _backward(K, N, dtype, ALL, ld, ld, 0, K + N, in_place=in_place)


@pytest.mark.parametrize("form", [dict(ALL, post=0), dict(ALL, pre=0), dict(ALL, gate=0, token=0), dict(post=0, gate=0, token=0, pre=1, block=0)],
                         ids=["no norm after", "no norm before", "no gates", "no block"])
def test_forms(form):
    for ls, lb in ((192, 192), (192, 256), (256, 192)):
        _forward(1100, 150, "bf16", form, ls, lb, 0, ls + lb)
        _backward(1100, 150, "bf16", form, ls, lb, 0, ls + lb)


@pytest.mark.parametrize("ls,lb", [(128, 136), (136, 128), (128, 131)])
def test_lines_on_one_side_alone(ls, lb):
    """One of the two leading dimensions is no multiple of 64: not this layout, and the same results."""
    for in_place in (False, True):
        _forward(1100, 120, "bf16", ALL, ls, lb, 0, ls, in_place=in_place)
        _backward(1100, 120, "bf16", ALL, ls, lb, 0, ls, in_place=in_place)
