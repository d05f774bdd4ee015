"""Dense layers and their gradients against the formulas in float64: small integers, whose sums are exact, bit for bit; real
values within a tolerance that counts roundings."""
import numpy as np
import pytest

from tests.dense_cases import SHAPES
from tests.dense_util import DEV, HALF, TORCH, Matrix, integers, result, rounded, workspace
from oracle import dense_oracle as orc

pytestmark = pytest.mark.gpu

FLAG = {"none": 0, "relu": 1, "gelu": 4, "gelu_tanh": 8, "silu": 16}
# how rows lie: (what is added to the least pitch of whole pieces, elements ahead of the matrix); None: rows follow one another
LAYOUTS = {"pieces": (0, 0), "apart": (24, 16), "anywhere": (None, 0), "odd": (3, 5)}


def _place(cols, layout):
    more, offset = LAYOUTS[layout]
    return (cols, 0) if more is None else ((cols + 7) // 8 * 8 + more, offset)


def _matrix(rows, cols, dtype, layout, values):
    ld, offset = _place(cols, layout)
    return Matrix(rows, cols, dtype, ld, offset, values)


def _result(rows, cols, dtype, layout):
    ld, offset = _place(cols, layout)
    return result(rows, cols, dtype, ld, offset)


def forward(hinm, W, X, dtype, bias=None, residual=None, keep=False, flags=0, layout="pieces", out=None, stream=None):
    """(Y, Z, W, X) as matrices; checks that nothing beside the results was written."""
    import torch
    (M, K), N = W.shape, X.shape[1]
    w, x = _matrix(M, K, dtype, layout, W), _matrix(K, N, dtype, layout, X)
    b = None if bias is None else torch.as_tensor(bias, dtype=torch.float32, device=DEV)
    r = None if residual is None else _matrix(M, N, dtype, layout, residual)
    y = _result(M, N, torch.float32 if flags & 2 else dtype, layout)
    z = _result(M, N, dtype, layout) if keep else None
    before = [m.surroundings() for m in (y, z) if m]
    ws = workspace(hinm.hinm_linear_workspace(M, K, N))
    hinm.hinm_linear(M, K, N, dtype, w.data, w.ld, x.data, x.ld, b, r.data if r else None, r.ld if r else 0, z.data if z else None, y.data,
                     y.ld, flags, *ws, stream=stream)
    torch.cuda.synchronize()
    for m, old in zip((m for m in (y, z) if m), before):
        assert torch.equal(m.surroundings(), old)
    return y, z, w, x


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("M,K,N", SHAPES)
def test_integers_forward(M, K, N, layout):
    import paper_2407_20496_amd as hinm
    rng = np.random.default_rng(M * 7 + K * 3 + N)
    dtype = ("f16", "bf16")[(M + N) % 2]
    W, X, R, b = integers(rng, M, K), integers(rng, K, N), integers(rng, M, N, 9), integers(rng, 1, M, 9)[0]
    y, z, _, _ = forward(hinm, W, X, dtype, b, R, True, FLAG["relu"], layout)
    want, wz = orc.linear(W, X, b, R, "relu")
    assert np.array_equal(z.f64(), rounded(wz, dtype))
    assert np.array_equal(y.f64(), rounded(want, dtype))
    y, _, _, _ = forward(hinm, W, X, dtype, flags=2, layout=layout)
    assert np.array_equal(y.f64(), W @ X)


def gradients(hinm, W, X, Z, dY, dtype, name="none", layout="pieces", f32=False, want=(True, True, True)):
    import torch
    (M, K), N = W.shape, X.shape[1]
    w, x, g = _matrix(M, K, dtype, layout, W), _matrix(K, N, dtype, layout, X), _matrix(M, N, dtype, layout, dY)
    z = _matrix(M, N, dtype, layout, Z) if Z is not None else None
    dx = _result(K, N, dtype, layout) if want[0] else None
    dw = _result(M, K, torch.float32 if f32 else dtype, layout) if want[1] else None
    db = torch.full((M + 1,), 77.0, device=DEV) if want[2] else None
    before = [m.surroundings() for m in (dx, dw) if m]
    ws = workspace(hinm.hinm_linear_grad_workspace(M, K, N))
    hinm.hinm_linear_grad(M, K, N, dtype, w.data, w.ld, x.data, x.ld, z.data if z else None, g.data, g.ld, dx.data if dx else None,
                          dw.data if dw else None, db, FLAG[name] | (2 if f32 else 0), *ws)
    torch.cuda.synchronize()
    for m, old in zip((m for m in (dx, dw) if m), before):
        assert torch.equal(m.surroundings(), old)
    assert db is None or db[M].item() == 77.0
    return dx, dw, None if db is None else db[:M].double().cpu().numpy()


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("M,K,N", SHAPES)
def test_integers_backward(M, K, N, layout):
    import paper_2407_20496_amd as hinm
    rng = np.random.default_rng(M * 5 + K + N * 11)
    dtype = ("f16", "bf16")[(K + N) % 2]
    W, X, Z, dY = integers(rng, M, K), integers(rng, K, N), integers(rng, M, N), integers(rng, M, N)
    name = ("none", "relu")[M % 2]
    dx, dw, db = gradients(hinm, W, X, Z, dY, dtype, name, layout, f32=K % 2 == 0)
    wx, ww, wb, _ = orc.linear_grad(W, X, Z, dY, name)
    assert np.array_equal(dx.f64(), rounded(wx, dtype))
    assert np.array_equal(dw.f64(), ww if K % 2 == 0 else rounded(ww, dtype))
    assert np.array_equal(db, wb)


@pytest.mark.parametrize("want", [(True, False, False), (False, True, False), (False, False, True), (True, False, True)])
def test_gradients_one_by_one(want):
    import paper_2407_20496_amd as hinm
    rng = np.random.default_rng(3)
    W, X, Z, dY = integers(rng, 70, 90), integers(rng, 90, 40), integers(rng, 70, 40), integers(rng, 70, 40)
    for name in ("none", "relu"):
        got = gradients(hinm, W, X, Z, dY, "bf16", name, want=want)
        for g, w, asked in zip(got, orc.linear_grad(W, X, Z, dY, name), want):
            assert (g is not None) == asked
            if asked:
                assert np.array_equal(g if isinstance(g, np.ndarray) else g.f64(), w if isinstance(g, np.ndarray) else rounded(w, "bf16"))


def _sum_error(A, B, half_of_operands=0.0):
    """How far a product in float32 may be from A B: an instruction adds 16 products, in some order, to a running sum, and the parts
    of a tile are added at the end (fewer than 24 of them): K / 16 + 16 + 24 roundings or cuts of at most 2^-23 of the sum of
    magnitudes; and what rounded operands bring."""
    S = np.abs(A) @ np.abs(B)
    return ((A.shape[1] / 16 + 40) * 2.0 ** -23 + half_of_operands) * S


@pytest.mark.parametrize("name", orc.ACTS)
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("M,K,N", [(96, 200, 1), (64, 512, 13), (200, 333, 150), (512, 1024, 257)])
def test_activations_forward(M, K, N, dtype, name):
    import paper_2407_20496_amd as hinm
    rng = np.random.default_rng(M + N)
    # some rows far out, where an activation's tail counts
    W = rng.normal(size=(M, K)) / np.sqrt(K) * np.where(np.arange(M) % 3 == 0, 4.0, 1.0)[:, None]
    X, b, R = rng.normal(size=(K, N)), rng.normal(size=M), rng.normal(size=(M, N))
    W, X, R = (rounded(v, dtype) for v in (W, X, R))
    b = b.astype(np.float32).astype(np.float64)
    for residual in (None, R):
        y, z, _, _ = forward(hinm, W, X, dtype, b, residual, True, FLAG[name])
        Y, Z = orc.linear(W, X, b, residual, name)
        off_z = _sum_error(W, X) + 2.0 ** -23 * (np.abs(Z) + np.abs(b)[:, None])
        # a smallest step of f16 is 2^-24
        assert (np.abs(z.f64() - Z) <= HALF[dtype] * (np.abs(Z) + off_z) + off_z + 2.0 ** -25).all()
        # slopes stay below 1.13; the activation itself is within 2^-20 of its value, and its argument's exponent is rounded
        off = 1.13 * off_z + 2.0 ** -20 * np.abs(Z) + 2.0 ** -23 * np.abs(Y)
        assert (np.abs(y.f64() - Y) <= HALF[dtype] * (np.abs(Y) + off) + off + 2.0 ** -25).all()


@pytest.mark.parametrize("name", orc.ACTS[1:])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("M,K,N", [(96, 200, 1), (64, 72, 513), (200, 333, 150)])
def test_activations_backward(M, K, N, dtype, name):
    import paper_2407_20496_amd as hinm
    rng = np.random.default_rng(M + N + 1)
    W, X, Z, dY = (rounded(rng.normal(size=s), dtype) for s in ((M, K), (K, N), (M, N), (M, N)))
    Z *= 4.0  # exact
    dx, dw, db = gradients(hinm, W, X, Z, dY, dtype, name)
    wx, ww, wb, dZ = orc.linear_grad(W, X, Z, dY, name)
    # dZ: its slope (of at most 1.13, beside a |z| times its own error) within 2^-19, and one rounding to the type
    off_slope = 2.0 ** -19 * np.abs(dY) * (1 + np.abs(Z))
    off_dz = HALF[dtype] * (np.abs(dZ) + off_slope) + off_slope + 2.0 ** -25
    for got, want, A, B, off in ((dx.f64(), wx, W.T, dZ, np.abs(W.T) @ off_dz), (dw.f64(), ww, dZ, X.T, off_dz @ np.abs(X.T))):
        off = off + _sum_error(np.abs(A), np.abs(B)) * 1.01
        assert (np.abs(got - want) <= HALF[dtype] * (np.abs(want) + off) + off + 2.0 ** -25).all()
    # sums of unrounded values: log-many and a few in a row, at most N / 64 + 16 additions deep
    assert (np.abs(db - wb) <= off_slope.sum(1) + (N / 64 + 16) * 2.0 ** -24 * np.abs(dZ).sum(1)).all()


@pytest.mark.parametrize("name", orc.ACTS[1:])
def test_gradients_are_differences(name):
    """dX, dW and dbias along random directions against differences of the float64 forward pass."""
    import paper_2407_20496_amd as hinm
    rng = np.random.default_rng(9)
    M, K, N = 48, 56, 24
    W, X, dY = (rounded(rng.normal(size=s) / 4, "f16") for s in ((M, K), (K, N), (M, N)))
    b = rng.normal(size=M)
    Z = rounded(W @ X + b[:, None], "f16")
    if name == "relu":
        # away from the corner at zero, where there is no derivative
        Z = np.where(np.abs(Z) < 0.01, 0.5, Z)
    dx, dw, db = gradients(hinm, W, X, Z, dY, "f16", name)
    for got, dz_of in ((dx.f64(), lambda d: W @ d), (dw.f64(), lambda d: d @ X), (db, lambda d: np.tile(d[:, None], (1, N)))):
        d = rng.normal(size=got.shape)
        h = 1e-5
        step = h * dz_of(d)
        slope = ((orc.act(Z + step, name) - orc.act(Z - step, name)) * dY).sum() / (2 * h)
        # every element of a gradient is off by two roundings of its terms at most: sqrt(n) of them beside their sum
        scale = np.sqrt((got ** 2 * d ** 2).sum())
        assert abs((got * d).sum() - slope) <= 8 * HALF["f16"] * scale + 1e-6 * np.abs(got * d).sum()


def test_far_out_and_not_finite():
    """Values at the ends of the activations, infinities and NaN: as the formulas have them, each row by itself."""
    import paper_2407_20496_amd as hinm
    far = np.array([-60000.0, -500.0, -40.0, -12.0, 0.0, 12.0, 40.0, 500.0, 60000.0])
    K = 8
    W = np.zeros((len(far), K))
    W[:, 0] = far
    X = np.zeros((K, 16))
    X[0] = 1
    for name in orc.ACTS:
        y, _, _, _ = forward(hinm, W, X, "bf16", flags=FLAG[name])
        want = rounded(orc.act(rounded(far, "bf16"), name), "bf16")
        got = y.f64()
        assert np.isfinite(got).all() and np.allclose(got, want[:, None], rtol=2.0 ** -7, atol=1e-30), name
        Z = np.tile(far[:, None], (1, 16))
        _, _, db = gradients(hinm, np.ones((len(far), 8)), np.ones((8, 16)), Z, np.ones((len(far), 16)), "bf16", name)
        assert np.allclose(db, 16 * orc.slope(rounded(far, "bf16"), name), rtol=1e-4, atol=1e-3), name
    W[3, 5] = np.inf
    W[5, 0] = np.nan
    X[5] = 1
    y, _, _, _ = forward(hinm, W, X, "bf16", flags=FLAG["relu"])
    got = y.f64()
    assert np.isposinf(got[3]).all() and np.isnan(got[5]).all()
    assert np.isfinite(np.delete(got, [3, 5], 0)).all()
    X[2, 7] = np.nan  # one token's input
    got = forward(hinm, W, X, "bf16")[0].f64()
    assert np.isnan(got[:, 7]).all() and np.isfinite(np.delete(np.delete(got, [3, 5], 0), 7, 1)).all()


@pytest.mark.parametrize("M,K,N", [(130, 100, 1), (256, 512, 16), (384, 1024, 200), (64, 64, 9)])
@pytest.mark.parametrize("layout", ["pieces", "odd"])
def test_sum_in_place(M, K, N, layout):
    import torch
    import paper_2407_20496_amd as hinm
    rng = np.random.default_rng(K)
    W, X, H = integers(rng, M, K), integers(rng, K, N), integers(rng, M, N, 9)
    w, x, h = _matrix(M, K, "bf16", layout, W), _matrix(K, N, "bf16", layout, X), _matrix(M, N, "bf16", layout, H)
    before = h.surroundings()
    hinm.hinm_linear(M, K, N, "bf16", w.data, w.ld, x.data, x.ld, None, h.data, h.ld, None, h.data, h.ld, 0,
                     *workspace(hinm.hinm_linear_workspace(M, K, N)))
    torch.cuda.synchronize()
    assert torch.equal(before, h.surroundings())
    assert np.array_equal(h.f64(), rounded(W @ X + H, "bf16"))


@pytest.mark.parametrize("M,K,N", [(256, 512, 1), (256, 4096, 16), (300, 1000, 200), (768, 768, 512)])
def test_same_call_same_bits_on_any_stream_and_in_graphs(M, K, N):
    import torch
    import paper_2407_20496_amd as hinm
    gen = torch.Generator(device=DEV)
    gen.manual_seed(5)
    new = lambda r, c: torch.randn(r, c, device=DEV, generator=gen).bfloat16()
    ld = N if N == 1 else (N + 7) // 8 * 8
    W, X, dY, Z = new(M, K), new(K, ld), new(M, ld), new(M, ld)
    Y, dX, dW, db = (torch.empty_like(Z), torch.empty_like(X), torch.empty_like(W), torch.empty(M, device=DEV))
    ws = workspace(max(hinm.hinm_linear_workspace(M, K, N), hinm.hinm_linear_grad_workspace(M, K, N)))

    def step(stream=None):
        hinm.hinm_linear(M, K, N, "bf16", W, K, X, ld, None, None, 0, Z, Y, ld, hinm.EPI_GELU, *ws, stream=stream)
        hinm.hinm_linear_grad(M, K, N, "bf16", W, K, X, ld, Z, dY, ld, dX, dW, db, hinm.EPI_GELU, *ws, stream=stream)

    outputs = lambda: [t[:, :N].clone() if t.dim() == 2 and t is not dW else t.clone() for t in (Y, Z, dX, dW, db)]
    step()
    torch.cuda.synchronize()
    want = outputs()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    step(stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outputs(), want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for t in (Y, dX, dW, db):
            t.fill_(7)
        ws[0].fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outputs(), want))


@pytest.mark.parametrize("pitch", [(1 << 21) - 8, (1 << 21) + 8])
def test_offsets_beyond_32_bits(pitch):
    """Rows so far apart that the last ones lie beyond 2^31 elements, on both sides of what a stage's copies can reach."""
    import torch
    import paper_2407_20496_amd as hinm
    rng = np.random.default_rng(2)
    M, K, N = 1100, 1096, 40
    W, X, dY = integers(rng, M, K), integers(rng, K, N), integers(rng, M, N)
    whole = torch.empty(M * pitch, dtype=torch.bfloat16, device=DEV)
    view = whole.as_strided((M, K), (pitch, 1))
    view.copy_(torch.as_tensor(W, device=DEV).bfloat16())
    x = Matrix(K, N, "bf16", values=X)
    y = result(M, N, "bf16")
    hinm.hinm_linear(M, K, N, "bf16", whole, pitch, x.data, x.ld, None, None, 0, None, y.data, y.ld, 0,
                     *workspace(hinm.hinm_linear_workspace(M, K, N)))
    assert np.array_equal(y.f64(), rounded(W @ X, "bf16"))
    g = Matrix(M, N, "bf16", values=dY)
    dx = result(K, N, "bf16")
    hinm.hinm_linear_grad(M, K, N, "bf16", whole, pitch, x.data, x.ld, None, g.data, g.ld, dx.data, None, None, 0,
                          *workspace(hinm.hinm_linear_grad_workspace(M, K, N)))
    assert np.array_equal(dx.f64(), rounded(W.T @ dY, "bf16"))
    # ... and a result there
    hinm.hinm_linear_grad(M, K, N, "bf16", None, pitch, x.data, x.ld, None, g.data, g.ld, None, whole, None, 0,
                          *workspace(hinm.hinm_linear_grad_workspace(M, K, N)))
    assert np.array_equal(view.double().cpu().numpy(), rounded(dY @ X.T, "bf16"))
