"""Every form of a dense layer's products at sizes that reach it, on integers whose sums are exact: whole and cut stages, fewer and
more of them than a ring holds, tiles that several workgroups share, weights that are copied first.  That a size reaches its form is
asked of a plan, on the CPU."""
import re

import pytest

LARGE, WIDE, MIDDLE, SMALL = (4, 4), (4, 2), (2, 2), (1, 1)
# (which: 0 the layer, 1 its input's gradient, 2 its weights'; M, K, N; tiles of a wave; shared; aligned weights)
TILES = [
    (0, 2617, 360, 11959, LARGE, True, True), (0, 7600, 64, 1145, LARGE, False, True), (0, 2564, 70, 3088, LARGE, False, True),
    (0, 5610, 144, 1609, LARGE, False, True), (0, 1573, 305, 5098, LARGE, False, True), (0, 7552, 1, 1218, LARGE, False, True),
    (0, 3462, 11944, 144, WIDE, True, True), (0, 131, 8444, 4138, WIDE, True, True), (0, 11528, 8, 322, WIDE, False, True),
    (0, 1356, 64, 2988, WIDE, False, True), (0, 386, 72, 10649, WIDE, False, True), (0, 2773, 132, 1605, WIDE, False, True),
    (0, 357, 203, 11046, WIDE, False, True), (0, 966, 320, 4717, WIDE, False, True),
    (0, 66, 6529, 3561, MIDDLE, True, True), (0, 10189, 2688, 83, MIDDLE, True, True), (0, 241, 1, 8432, MIDDLE, False, True),
    (0, 584, 64, 3502, MIDDLE, False, True), (0, 131, 80, 10913, MIDDLE, False, True), (0, 167, 134, 11125, MIDDLE, False, True),
    (0, 130, 247, 11022, MIDDLE, False, True), (0, 7245, 312, 320, MIDDLE, False, True),
    (1, 11040, 1606, 2700, LARGE, True, True), (1, 8, 5472, 1519, LARGE, False, True), (1, 65, 899, 9618, LARGE, False, True),
    (1, 139, 7300, 1180, LARGE, False, True), (1, 263, 1268, 6529, LARGE, False, True),
    (1, 5002, 132, 5702, WIDE, True, True), (1, 64, 6367, 675, WIDE, False, True), (1, 66, 10433, 405, WIDE, False, True),
    (1, 134, 3601, 1274, WIDE, False, True), (1, 205, 455, 8449, WIDE, False, True),
    (1, 5676, 2908, 65, MIDDLE, True, True), (1, 1, 223, 9225, MIDDLE, False, True), (1, 88, 2546, 856, MIDDLE, False, True),
    (1, 130, 328, 5829, MIDDLE, False, True), (1, 224, 7196, 372, MIDDLE, False, True), (1, 704, 152, 11330, MIDDLE, False, True),
    (2, 9309, 3471, 367, LARGE, True, True), (2, 4098, 968, 64, WIDE, False, True), (2, 7097, 602, 72, WIDE, False, True),
    (2, 6152, 136, 5611, WIDE, True, True), (2, 1688, 2650, 132, WIDE, False, True), (2, 1707, 2799, 58, WIDE, False, True),
    (2, 96, 1355, 10882, MIDDLE, True, True), (2, 1054, 2013, 64, MIDDLE, False, True), (2, 9977, 193, 68, MIDDLE, False, True),
    (2, 271, 6551, 152, MIDDLE, False, True), (2, 334, 9756, 256, MIDDLE, False, True), (2, 11561, 134, 299, MIDDLE, False, True),
    (0, 4097, 4097, 600, MIDDLE, False, False), (1, 4097, 4097, 600, MIDDLE, False, False), (0, 700, 30, 1030, SMALL, False, False),
    (0, 31, 2500, 250, SMALL, True, False), (1, 5, 33, 300, SMALL, False, False)]
# both gradients in one launch, of fewer and more workgroups than a chip holds; M, K, N; tiles of a wave
PAIRS = [(21, 16, 64, SMALL), (64, 2697, 101, SMALL), (128, 687, 144, SMALL), (166, 178, 205, SMALL), (188, 3263, 3596, SMALL), (384, 573, 4603, SMALL),
         (371, 4802, 64, SMALL), (106, 201, 9, SMALL), (2487, 2992, 9, SMALL), (282, 3880, 98, SMALL), (3615, 1628, 239, SMALL), (2752, 520, 840, SMALL),
         (1, 1, 1, SMALL), (170, 4632, 1855, MIDDLE), (320, 3138, 3369, MIDDLE), (231, 5318, 167, MIDDLE), (4104, 5315, 195, MIDDLE), (2050, 2048, 1024, MIDDLE)]
# weights' gradients of few tokens; M, K, N
OUTER = [(872, 4775, 1), (1, 1, 1), (64, 512, 32), (128, 1024, 8), (65, 513, 7), (63, 511, 9), (200, 129, 16), (17, 8, 31), (1, 700, 17), (513, 1, 5), (1000, 1000, 3),
         (96, 2056, 24)]
FEW = [(10300, 100, 9, 4), (10300, 200, 16, 4), (300, 1030, 16, 1), (257, 64, 2, 1)]


@pytest.mark.parametrize("which,M,K,N,tiles,shared,aligned", TILES)
def test_a_size_reaches_its_form(which, M, K, N, tiles, shared, aligned):
    import paper_2407_20496_amd as hinm
    text = hinm.hinm_calib_linear_plan(M, K, N, "f16", which, aligned)
    assert "WM=%d,WN=%d," % tiles in text and "GUARDED=0" in text, text
    assert ("linear_join_kernel" in text) == shared and (int(re.search(r"splits=(\d+)", text).group(1)) > 1) == shared
    assert ("linear_copy_kernel" in text) == (not aligned)


@pytest.mark.parametrize("M,K,N,blocks", FEW)
def test_few_tokens_reach_their_form(M, K, N, blocks):
    import paper_2407_20496_amd as hinm
    assert "linear_few_kernel" in hinm.hinm_calib_linear_plan(M, K, N, "f16") and "RB=%d," % blocks in hinm.hinm_calib_linear_plan(M, K, N, "f16")
    assert "PIECES=0" in hinm.hinm_calib_linear_plan(M, K, N, "f16", 0, False)


@pytest.mark.parametrize("M,K,N,tiles", PAIRS)
def test_both_gradients_reach_one_launch(M, K, N, tiles):
    import paper_2407_20496_amd as hinm
    text = hinm.hinm_calib_linear_plan(M, K, N, "bf16", 3)
    assert text.startswith("linear_pair_kernel<") and "WM=%d,WN=%d>" % tiles in text and ";" not in text.strip("; \n"), text
    apart = hinm.hinm_calib_linear_plan(4096, 4096, 2048, "bf16", 3)
    assert "pair" not in apart and apart.count("linear_tile_kernel") == 2


def _integers(rows, cols, gen, most=2):
    import torch
    return torch.randint(-most, most + 1, (rows, cols), device="cuda:0", generator=gen).double()


@pytest.mark.gpu
@pytest.mark.parametrize("which,M,K,N,aligned", [(*t[:4], t[6]) for t in TILES] + [(0, *f[:3], a) for f in FEW for a in (True, False)])
def test_products_of_integers(which, M, K, N, aligned):
    import torch
    import paper_2407_20496_amd as hinm
    from tests.dense_util import Matrix, result, workspace
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(M + K + N)
    dtype = ("f16", "bf16")[K % 2]
    W, X, G = _integers(M, K, gen), _integers(K, N, gen), _integers(M, N, gen)
    w = Matrix(M, K, dtype, None if aligned else K, 0 if aligned else 1, W)
    x, g = Matrix(K, N, dtype, values=X), Matrix(M, N, dtype, values=G)
    real = lambda v: v.to(w.kind).double()  # sums below 2^24 are exact in float32, so one rounding is left
    if which == 0:
        y = result(M, N, dtype)
        around = y.surroundings()
        hinm.hinm_linear(M, K, N, dtype, w.data, w.ld, x.data, x.ld, None, g.data, g.ld, None, y.data, y.ld, 0,
                         *workspace(hinm.hinm_linear_workspace(M, K, N)))
        out, want = y, real(W @ X + G)
    else:
        out = result(K, N, dtype) if which == 1 else result(M, K, dtype, w.ld, w.offset)
        around = out.surroundings()
        hinm.hinm_linear_grad(M, K, N, dtype, w.data, w.ld, x.data, x.ld, None, g.data, g.ld, out.data if which == 1 else None,
                              out.data if which == 2 else None, None, 0, *workspace(hinm.hinm_linear_grad_workspace(M, K, N)))
        want = real(W.t().contiguous() @ G) if which == 1 else real(G @ X.t().contiguous())
    torch.cuda.synchronize()
    assert torch.equal(out.view.double(), want)
    assert torch.equal(out.surroundings(), around)


@pytest.mark.gpu
@pytest.mark.parametrize("act", [False, True])
@pytest.mark.parametrize("M,K,N", [p[:3] for p in PAIRS])
def test_both_gradients_of_integers(M, K, N, act):
    """With relu as the activation, whose slopes are 0 and 1; rows have numbers behind their ends that are no part of a sum."""
    import torch
    import paper_2407_20496_amd as hinm
    from tests.dense_util import Matrix, result, workspace
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(M + K + N)
    dtype = ("f16", "bf16")[M % 2]
    W, X, G, Z = _integers(M, K, gen), _integers(K, N, gen), _integers(M, N, gen), _integers(M, N, gen)
    w, x, g, z = (Matrix(*v.shape, dtype, values=v) for v in (W, X, G, Z))
    dx, dw, db = result(K, N, dtype), result(M, K, dtype), torch.full((M + 1,), 77.0, device="cuda:0")
    around = dx.surroundings(), dw.surroundings()
    hinm.hinm_linear_grad(M, K, N, dtype, w.data, w.ld, x.data, x.ld, z.data if act else None, g.data, g.ld, dx.data, dw.data, db,
                          hinm.EPI_RELU if act else 0, *workspace(hinm.hinm_linear_grad_workspace(M, K, N)))
    torch.cuda.synchronize()
    if act:
        G = torch.where(Z > 0, G, 0.0)
    real = lambda v: v.to(w.kind).double()
    assert torch.equal(torch.as_tensor(dx.f64(), device="cuda:0"), real(W.t().contiguous() @ G))
    assert torch.equal(torch.as_tensor(dw.f64(), device="cuda:0"), real(G @ X.t().contiguous()))
    assert torch.equal(db[:M].double(), G.sum(1)) and db[M].item() == 77.0
    assert torch.equal(dx.surroundings(), around[0]) and torch.equal(dw.surroundings(), around[1])


@pytest.mark.parametrize("M,K,N", OUTER)
def test_few_tokens_reach_their_gradient(M, K, N):
    import paper_2407_20496_amd as hinm
    for aligned in (True, False):
        assert hinm.hinm_calib_linear_plan(M, K, N, "f16", 2, aligned).startswith("linear_outer_kernel")
    assert "outer" not in hinm.hinm_calib_linear_plan(M, K, 33, "f16", 2)


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["pieces", "odd", "close"])
@pytest.mark.parametrize("out", ["same", "f32"])
@pytest.mark.parametrize("M,K,N", OUTER)
def test_weights_gradient_of_few_tokens(M, K, N, out, layout):
    """Integers, whose sums are exact; rows have NaN behind and around them."""
    import torch
    import paper_2407_20496_amd as hinm
    from tests.dense_util import Matrix, pitch8, result, workspace
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(M + K + N)
    dtype = ("f16", "bf16")[K % 2]
    X, G = _integers(K, N, gen, 7), _integers(M, N, gen, 7)
    place = {"pieces": lambda n: (pitch8(n), 0), "odd": lambda n: (n + 3, 5), "close": lambda n: (n, 1)}[layout]
    x, g = Matrix(K, N, dtype, *place(N), X), Matrix(M, N, dtype, *place(N), G)
    dw = result(M, K, torch.float32 if out == "f32" else dtype, *place(K))
    around = dw.surroundings()
    hinm.hinm_linear_grad(M, K, N, dtype, None, dw.ld, x.data, x.ld, None, g.data, g.ld, None, dw.data, None,
                          hinm.OUT_F32 if out == "f32" else 0, *workspace(hinm.hinm_linear_grad_workspace(M, K, N)))
    torch.cuda.synchronize()
    assert torch.equal(dw.view.double(), (G @ X.t().contiguous()).to(dw.kind).double())
    assert torch.equal(dw.surroundings(), around)
