"""Every form of the 4-bit product at sizes that its estimates send there: rows, columns and lines of 256 that do not fill their
tiles, odd and even counts of lines, one line, matrices narrower than a tile.

Which form serves which size is asked of the library on the CPU, so that other estimates cannot leave a form untested unseen."""
import numpy as np
import pytest

from oracle import block_oracle as orc
from tests.test_gpu_mx4 import DEV, GUARD, _draw, _form, _guarded, _matrix, _tolerance, _wide

STREAM = "mx4_stream_kernel<OUT={},WM=%d,WN=%d,WAVES=%d>"
TILE = "mx4_tile_kernel<OUT={},WM=%d,WN=%d,RING=%d>"
FORMS = {   # M, N, K
    STREAM % (1, 1, 8): [(130, 129, 4100)],
    STREAM % (1, 2, 8): [(37, 4252, 1305), (6506, 33, 1047), (1, 16476, 2100)],
    STREAM % (2, 2, 8): [(15089, 2, 1080), (34, 13137, 1043), (1030, 770, 1160)],
    STREAM % (2, 4, 4): [(13214, 25, 984), (34, 16457, 611), (267, 17055, 84)],
    TILE % (2, 2, 4): [(65, 16563, 986), (1255, 1581, 1030), (66, 17515, 2123)],
    TILE % (2, 2, 2): [(13838, 67, 18), (67, 16606, 317), (11521, 140, 525), (2561, 2563, 1030), (2561, 2563, 2310)],
    TILE % (4, 4, 2): [(2999, 3001, 4100), (5000, 4999, 1281)],
}
SHAPES = [s for v in FORMS.values() for s in v]
ONE_EACH = [(37, 4252, 1305), (1030, 770, 1160), (34, 16457, 611), (1255, 1581, 1030), (11521, 140, 525), (5000, 4999, 1281)]
TILES = {(1255, 1581, 1030): TILE % (2, 2, 4), (11521, 140, 525): TILE % (2, 2, 2), (5000, 4999, 1281): TILE % (4, 4, 2)}


def test_the_sizes_reach_every_form():
    import paper_2407_20496_amd as hinm
    assert [sum(s in v for s in ONE_EACH) for v in FORMS.values()] == [0, 1, 1, 1, 1, 1, 1]
    assert [sum(s in v for s in TILES) for v in FORMS.values()] == [0, 0, 0, 0, 1, 1, 1]
    for form, shapes in FORMS.items():
        for M, N, K in shapes:
            for out, flags, dtype in ((0, 0, "f16"), (1, hinm.EPI_RELU, "bf16"), (2, hinm.OUT_F32, "f16")):
                plan = hinm.hinm_calib_mx4_plan(M, N, K, dtype, flags)
                assert plan.startswith(form.format(out)), (M, N, K, plan)
    for (M, N, K), form in TILES.items():
        plan = hinm.hinm_calib_mx4_plan(M, N, K, "bf16", 0, True)
        assert plan.startswith("mx4_columns_kernel<DT=1>; " + form.format(1)), plan
    # and the forms that quantise on their way
    for (M, K, N), name in {(300, 4096, 1): "mx4_token_kernel<OUT=1,DT=1>", (70, 1000, 8): "mx4_few_kernel<OUT=1,DT=1,P=1>",
                            (70, 1000, 16): "mx4_few_kernel<OUT=1,DT=1,P=2>", (64, 333, 40): "mx4_few_kernel<OUT=1,DT=1,P=4>"}.items():
        assert hinm.hinm_calib_mx4_plan(M, N, K, "bf16", 0, True).startswith(name)


def test_what_a_plan_refuses():
    import ctypes as C
    import paper_2407_20496_amd as hinm
    lib, text = hinm.load_library(), C.create_string_buffer(b"x" * 40)
    assert lib.hinm_calib_mx4_plan(64, 64, 64, 0, 0, 0, None, 40) == 1
    assert lib.hinm_calib_mx4_plan(64, 64, 64, 0, 0, 0, text, 0) == 1
    assert lib.hinm_calib_mx4_plan(0, 64, 64, 0, 0, 0, text, 40) == 2 and text.value == b""
    assert lib.hinm_calib_mx4_plan(64, 64, 64, 2, 0, 0, text, 40) == 3
    assert lib.hinm_calib_mx4_plan(64, 64, 64, 0, 4, 0, text, 40) == 5
    assert lib.hinm_calib_mx4_plan(16, 65, 1 << 30, 0, 0, 1, text, 40) == 5
    assert lib.hinm_calib_mx4_plan(64, 64, 64, 0, 0, 0, text, 12) == 0 and text.value == b"mx4_stream_"


def _random(rows, length, seed, low, high):
    """A random form, its padding as the quantiser leaves it."""
    rng = np.random.default_rng(seed)
    nib = np.zeros((rows, 2 * orc.code_pitch(length)), dtype=np.uint8)
    nib[:, :length] = rng.integers(0, 16, (rows, length), dtype=np.uint8)
    codes = nib[:, 0::2] | nib[:, 1::2] << 4
    scales = np.full((rows, orc.scale_pitch(length)), 127, dtype=np.uint8)
    for j in range((length + 31) // 32):
        scales[:, orc.scale_place(j)] = rng.integers(low, high, rows)
    return codes, scales


def _upload(form):
    import torch
    return tuple(torch.from_numpy(a).to(DEV) for a in orc.to_memory(*form, 0xFF))


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_product(M, N, K):
    import torch
    import paper_2407_20496_amd as hinm
    fa, fb = _random(M, K, M + 2 * N + 3 * K, 118, 130), _random(N, K, 5 * M + N + K, 120, 128)
    plain, size = orc.product(orc.values(*fa, K), orc.values(*fb, K))
    a, b = _upload(fa), _upload(fb)
    for out, relu, ld, first in (("f32", False, N, 0), ("f32", True, N + 1, 1), ("f16", True, N + 1, 1), ("bf16", False, (N + 7) // 8 * 8, 0)):
        want = np.maximum(plain, 0) if relu else plain
        Y = torch.full((first + M * ld + 16,), 0x4321, dtype=torch.float32 if out == "f32" else torch.int16, device=DEV)
        flags = (hinm.EPI_RELU if relu else 0) | (hinm.OUT_F32 if out == "f32" else 0)
        hinm.hinm_mx4_product(M, N, K, "f16" if out == "f32" else out, *a, *b, Y.data_ptr() + first * Y.element_size(), ld, flags)
        host = Y.cpu().numpy()
        rows = host[first:first + M * ld].reshape(M, ld)
        got = rows[:, :N].astype(np.float64) if out == "f32" else _wide(rows[:, :N].copy().view(np.uint16), out)
        fits = np.abs(want) < (65000 if out == "f16" else 1e30)
        assert fits.mean() > 0.99
        assert (np.abs(got - want) <= _tolerance(size, K, want, out))[fits].all(), (out, ld)
        assert (rows[:, N:] == 0x4321).all() and (host[:first] == 0x4321).all() and (host[first + M * ld:] == 0x4321).all(), (out, ld)


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", ONE_EACH)
def test_a_row_that_is_no_number_spoils_its_outputs_alone(M, N, K):
    import torch
    import paper_2407_20496_amd as hinm
    fa, fb = _random(M, K, 1, 118, 130), _random(N, K, 2, 120, 128)
    for f, row, block in ((fa, M - 1, 3), (fb, N // 2 + 1, (K - 1) // 32)):
        f[1][row, orc.scale_place(block)] = 255
        f[0][row, 16 * block:16 * block + 16] = 0
    nan = np.zeros((M, N), dtype=bool)
    nan[M - 1], nan[:, N // 2 + 1] = True, True
    for flags in (hinm.OUT_F32, hinm.OUT_F32 | hinm.EPI_RELU):
        Y = torch.zeros((M, N), dtype=torch.float32, device=DEV)
        hinm.hinm_mx4_product(M, N, K, "bf16", *_upload(fa), *_upload(fb), Y, N, flags)
        assert np.array_equal(torch.isnan(Y).cpu().numpy(), nan)


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", ONE_EACH)
def test_scales_at_their_ends(M, N, K):
    """2^-127 and 2^127 in one product: their factors cancel."""
    import torch
    import paper_2407_20496_amd as hinm
    fa, fb = _random(M, K, 3, 0, 1), _random(N, K, 4, 254, 255)
    want, size = orc.product(orc.values(*fa, K), orc.values(*fb, K))
    Y = torch.empty((M, N), dtype=torch.float32, device=DEV)
    hinm.hinm_mx4_product(M, N, K, "bf16", *_upload(fa), *_upload(fb), Y, N, hinm.OUT_F32)
    assert (np.abs(Y.cpu().numpy() - want) <= _tolerance(size, K, want, "f32")).all()


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", TILES)
def test_linear_is_quantize_and_product(M, N, K):
    import torch
    import paper_2407_20496_amd as hinm
    dtype = "bf16"
    w = _upload(_random(M, K, 11, 118, 130))
    bits = _draw(K, min(N, 700), dtype, 12)
    bits = np.ascontiguousarray(np.tile(bits, (1, (N + 699) // 700))[:, :N])
    for ld, first in ((N + 1, 1), ((N + 7) // 8 * 8, 0)):
        keep, X = _matrix(bits, ld, first)
        x = _form(N, K)
        hinm.hinm_mx4_quantize(K, N, dtype, X, ld, hinm.MX4_COLUMNS, *x)
        nbytes = hinm.hinm_mx4_linear_workspace(M, K, N)
        for flags, kind in ((0, torch.int16), (hinm.EPI_RELU | hinm.OUT_F32, torch.int32)):
            want, got, ws = torch.zeros((M, N), dtype=kind, device=DEV), torch.full((M, N), 77, dtype=kind, device=DEV), _guarded(nbytes)
            hinm.hinm_mx4_product(M, N, K, dtype, *w, *x, want, N, flags)
            hinm.hinm_mx4_linear(M, K, N, dtype, *w, X, ld, got, N, flags, ws, nbytes)
            assert torch.equal(got, want) and (ws[nbytes:] == GUARD).all(), (ld, flags)
        del keep


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", TILES)
def test_replays(M, N, K):
    """Three replays of a captured product on operands that change between them, with the program's own work around them."""
    import torch
    import paper_2407_20496_amd as hinm
    draws = [(_upload(_random(M, K, 20 + s, 118, 130)), _upload(_random(N, K, 30 + s, 120, 128))) for s in range(3)]
    a, b = ([t.clone() for t in f] for f in draws[0])
    Y, want = (torch.empty((M, N), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    call = lambda out: hinm.hinm_mx4_product(M, N, K, "bf16", *a, *b, out, N)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(Y)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            call(Y)
    torch.cuda.current_stream().wait_stream(side)
    for da, db in draws:
        for to, new in zip((*a, *b), (*da, *db)):
            to.copy_(new)
        call(want)
        Y.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(Y.view(torch.int16), want.view(torch.int16))
