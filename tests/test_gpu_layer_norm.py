"""Layer norm and its gradients against the formulas in float64."""
import numpy as np
import pytest

from tests.dense_util import DEV, HALF, Matrix, result, rounded, workspace
from oracle import dense_oracle as orc

pytestmark = pytest.mark.gpu

LAYOUTS = {"pieces": (0, 0), "lines": (None, 0), "odd": (3, 5), "close": (-1, 0)}
# one channel, one token, vectors, columns held by one workgroup, strips; row ends of every kind
SHAPES = [(1, 1), (1, 9), (9, 1), (4096, 1), (8000, 1), (16384, 1), (16390, 1), (20000, 1), (768, 7), (768, 130), (1024, 65), (4096, 16),
          (4096, 17), (2048, 8), (2050, 8), (1100, 129), (5000, 63), (1025, 64), (3001, 200), (64, 5000),
          (1500, 256), (2048, 41), (1024, 2048), (1024, 2049), (700, 4493), (4096, 5)]


def _place(cols, layout):
    more, offset = LAYOUTS[layout]
    if more is None:
        return (cols + 63) // 64 * 64, 0
    return (cols, 0) if more < 0 else ((cols + 7) // 8 * 8 + more, offset)


def _matrix(v, dtype, layout):
    ld, offset = (1, 0) if v.shape[1] == 1 and layout in ("close", "pieces") else _place(v.shape[1], layout)
    return Matrix(*v.shape, dtype, ld, offset, v)


def _result(K, N, dtype, layout):
    ld, offset = (1, 0) if N == 1 and layout in ("close", "pieces") else _place(N, layout)
    return result(K, N, dtype, ld, offset)


def _vector(v):
    import torch
    return None if v is None else torch.as_tensor(v, dtype=torch.float32, device=DEV)


def _f32(v):
    return v.astype(np.float32).astype(np.float64)


def _stream_values(rng, K, N, dtype):
    """A residual stream: channels of very different sizes, tokens with a mean."""
    return rounded((rng.normal(size=(K, N)) + 0.5) * np.exp(rng.normal(size=(K, 1))), dtype)


def forward(hinm, x, w, b, eps, dtype, layout="pieces", in_place=False):
    import torch
    K, N = x.shape
    m = _matrix(x, dtype, layout)
    u = m if in_place else _result(K, N, dtype, layout)
    mean, rstd = torch.full((N + 1,), 77.0, device=DEV), torch.full((N + 1,), 77.0, device=DEV)
    before = u.surroundings()
    hinm.hinm_layer_norm(K, N, dtype, eps, m.data, m.ld, _vector(w), _vector(b), u.data, u.ld, mean, rstd,
                         *workspace(hinm.hinm_layer_norm_workspace(K, N)))
    torch.cuda.synchronize()
    assert torch.equal(u.surroundings(), before) and mean[N].item() == 77.0 and rstd[N].item() == 77.0
    return u.f64(), mean[:N].double().cpu().numpy(), rstd[:N].double().cpu().numpy()


def _check_forward(got, x, w, b, eps, dtype):
    u, mean, rstd = got
    U, M, R = orc.layer_norm(x, w, b, eps)
    K = x.shape[0]
    spread = np.abs(x - M).mean(0) + np.abs(x).mean(0)
    # a workgroup adds at most K / 512 + 16 values in a row in float32, each to 2^-24 of the sum of magnitudes
    deep = (K / 512 + 20) * 2.0 ** -24
    off_mean = deep * np.abs(x).mean(0) + 2.0 ** -24 * np.abs(M)
    assert (np.abs(mean - M) <= off_mean).all()
    # the variance: the same depth, and the mean's error squared (first order cancels) ; the root halves it
    off_rstd = R * (deep + 4 * 2.0 ** -24 + off_mean ** 2 * R ** 2 + off_mean * R * 2.0 ** -20)
    assert (np.abs(rstd - R) <= off_rstd).all()
    W = 1.0 if w is None else np.abs(w)[:, None]
    off = W * (off_mean * R + np.abs(x - M) * off_rstd + 4 * 2.0 ** -24 * np.abs(x - M) * R) + 2.0 ** -23 * np.abs(U)
    if b is not None:
        off = off + 2.0 ** -24 * np.abs(b)[:, None]
    assert (np.abs(u - U) <= HALF[dtype] * (np.abs(U) + off) + off + 2.0 ** -25).all()
    assert np.isfinite(spread).all()


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("K,N", SHAPES)
def test_forward(K, N, layout):
    import paper_2407_20496_amd as hinm
    rng = np.random.default_rng(K + N)
    dtype = ("f16", "bf16")[(K + N) % 2]
    x = _stream_values(rng, K, N, dtype)
    w, b = _f32(1 + 0.3 * rng.normal(size=K)), _f32(rng.normal(size=K))
    if K % 3 == 0:
        w = None
    if N % 3 == 0:
        b = None
    _check_forward(forward(hinm, x, w, b, 1e-5, dtype, layout, in_place=N % 2 == 0), x, w, b, 1e-5, dtype)


@pytest.mark.parametrize("K,N", [(4096, 1), (700, 40), (3000, 70)])
@pytest.mark.parametrize("mean", [100.0, -3000.0])
def test_mean_far_beyond_the_deviations(K, N, mean):
    """f16 values around a mean of hundreds of their steps: nothing of the variance may be lost in the mean's square."""
    import paper_2407_20496_amd as hinm
    rng = np.random.default_rng(1)
    x = rounded(mean * (1 + rng.normal(size=(K, N)) * 2.0 ** -9), "f16")
    _check_forward(forward(hinm, x, None, None, 1e-5, "f16"), x, None, None, 1e-5, "f16")


@pytest.mark.parametrize("K,N", [(4096, 1), (700, 40), (3000, 70)])
def test_equal_channels(K, N):
    """No deviation at all: rstd is eps alone, u is b."""
    import paper_2407_20496_amd as hinm
    x = np.full((K, N), 3.0)
    b = _f32(np.linspace(-2, 2, K))
    u, mean, rstd = forward(hinm, x, None, b, 1e-5, "bf16")
    assert (mean == 3.0).all() and np.allclose(rstd, 1e-5 ** -0.5, rtol=2.0 ** -22)
    assert np.array_equal(u, np.tile(rounded(b, "bf16")[:, None], (1, N)))


@pytest.mark.parametrize("K,N", [(700, 40), (3000, 70)])
def test_not_finite_tokens_stay_by_themselves(K, N):
    import paper_2407_20496_amd as hinm
    rng = np.random.default_rng(4)
    x = _stream_values(rng, K, N, "bf16")
    y = x.copy()
    y[5, 3], y[K - 1, 17], y[0, 18] = np.inf, np.nan, -np.inf
    clean, broken = forward(hinm, x, None, None, 1e-5, "bf16"), forward(hinm, y, None, None, 1e-5, "bf16")
    bad = [3, 17, 18]
    assert np.isnan(broken[0][:, bad]).all() and np.isnan(broken[2][bad]).all()
    for a, b in zip(clean, broken):
        assert np.array_equal(np.delete(a, bad, -1), np.delete(b, bad, -1))


def backward(hinm, x, w, mean, rstd, du, dh, dtype, layout="pieces", want=(True, True, True), into=None):
    import torch
    K, N = x.shape
    mx, mu = _matrix(x, dtype, layout), _matrix(du, dtype, layout)
    mh = None if dh is None else _matrix(dh, dtype, layout)
    dx = {"dh": mh, "du": mu, None: _result(K, N, dtype, layout)}[into] if want[0] else None
    dw, db = (torch.full((K + 1,), 77.0, device=DEV) if asked else None for asked in want[1:])
    before = dx.surroundings() if dx else None
    hinm.hinm_layer_norm_grad(K, N, dtype, mx.data, mx.ld, _vector(w), _vector(mean), _vector(rstd), mu.data, mu.ld,
                              mh.data if mh else None, dx.data if dx else None, dw, db,
                              *workspace(hinm.hinm_layer_norm_grad_workspace(K, N)))
    torch.cuda.synchronize()
    assert dx is None or torch.equal(before, dx.surroundings())
    assert all(t is None or t[K].item() == 77.0 for t in (dw, db))
    host = lambda t: None if t is None else t[:K].double().cpu().numpy()
    return dx.f64() if dx else None, host(dw), host(db)


def _check_backward(got, x, w, mean, rstd, du, dh, dtype):
    DX, DW, DB = orc.layer_norm_grad(x, w, mean, rstd, du, dh)
    K, N = x.shape
    W = np.ones((K, 1)) if w is None else w[:, None]
    xn, g = (x - mean) * rstd, du * W
    e = 2.0 ** -24
    off_xn = 3 * e * (np.abs(xn) + np.abs(mean) * rstd)
    # sums down a column: at most K / 512 + 64 values or chunks in a row
    deep = (K / 512 + 80) * e
    off0 = (deep + 2 * e) * np.abs(g).mean(0)
    off1 = (deep + 4 * e) * np.abs(g * xn).mean(0) + (np.abs(g) * off_xn).mean(0)
    off = rstd * (2 * e * np.abs(g) + off0 + np.abs(xn) * off1 + (off_xn + 3 * e * np.abs(xn)) * np.abs((g * xn).mean(0))
                  + 4 * e * (np.abs(g) + np.abs(g).mean(0) + np.abs(xn * (g * xn).mean(0)))) + 2 * e * np.abs(DX)
    if dh is not None:
        off = off + 2 * e * np.abs(dh)
    dx, dw, db = got
    if dx is not None:
        assert (np.abs(dx - DX) <= HALF[dtype] * (np.abs(DX) + off) + off + 2.0 ** -25).all()
    deep = (N / 2048 + 64) * e
    if dw is not None:
        assert (np.abs(dw - DW) <= (deep + 3 * e) * np.abs(du * xn).sum(1) + (np.abs(du) * off_xn).sum(1)).all()
    if db is not None:
        assert (np.abs(db - DB) <= deep * np.abs(du).sum(1)).all()


def _backward_inputs(K, N, dtype, seed=0):
    rng = np.random.default_rng(K * 3 + N + seed)
    x, du, dh = _stream_values(rng, K, N, dtype), rounded(rng.normal(size=(K, N)), dtype), rounded(rng.normal(size=(K, N)), dtype)
    w = _f32(1 + 0.3 * rng.normal(size=K))
    _, mean, rstd = orc.layer_norm(x, w, None, 1e-5)
    return x, w, _f32(mean), _f32(rstd), du, dh


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("K,N", SHAPES)
def test_backward(K, N, layout):
    import paper_2407_20496_amd as hinm
    dtype = ("f16", "bf16")[(K + N) % 2]
    x, w, mean, rstd, du, dh = _backward_inputs(K, N, dtype)
    if K % 3 == 0:
        w = None
    if N % 2 == 0:
        dh = None
    _check_backward(backward(hinm, x, w, mean, rstd, du, dh, dtype, layout), x, w, mean, rstd, du, dh, dtype)


@pytest.mark.parametrize("K,N", [(64, 1), (768, 200), (3000, 70)])
@pytest.mark.parametrize("into", ["dh", "du"])
def test_backward_in_place(K, N, into):
    import paper_2407_20496_amd as hinm
    x, w, mean, rstd, du, dh = _backward_inputs(K, N, "bf16", 1)
    _check_backward(backward(hinm, x, w, mean, rstd, du, dh, "bf16", into=into), x, w, mean, rstd, du, dh, "bf16")


@pytest.mark.parametrize("K,N", [(300, 6), (768, 200), (3000, 70)])
@pytest.mark.parametrize("want", [(True, False, False), (False, True, False), (False, False, True)])
def test_backward_one_by_one(K, N, want):
    import paper_2407_20496_amd as hinm
    x, w, mean, rstd, du, dh = _backward_inputs(K, N, "f16", 2)
    got = backward(hinm, x, w, mean, rstd, du, dh, "f16", want=want)
    assert tuple(g is not None for g in got) == want
    _check_backward(got, x, w, mean, rstd, du, dh, "f16")


def test_backward_is_a_difference():
    """Along random directions against differences of the float64 forward pass."""
    import paper_2407_20496_amd as hinm
    K, N, eps, h = 200, 24, 1e-5, 1e-5
    x, w, _, _, du, _ = _backward_inputs(K, N, "f16", 3)
    _, mean, rstd = orc.layer_norm(x, w, None, eps)
    dx, dw, db = backward(hinm, x, w, mean, rstd, du, None, "f16")
    rng = np.random.default_rng(8)
    b = np.zeros(K)
    loss = lambda x, w, b: (orc.layer_norm(x, w, b, eps)[0] * du).sum()
    for got, of in ((dx, lambda d, s: loss(x + s * d, w, b)), (dw, lambda d, s: loss(x, w + s * d, b)), (db, lambda d, s: loss(x, w, b + s * d))):
        d = rng.normal(size=got.shape)
        slope = (of(d, h) - of(d, -h)) / (2 * h)
        scale = np.sqrt(((got * d) ** 2).sum())  # of roundings that are independent of one another
        assert abs((got * d).sum() - slope) <= 8 * HALF["f16"] * scale + 1e-6 * np.abs(got * d).sum()


@pytest.mark.parametrize("K,N", [(4096, 1), (768, 100), (3000, 130)])
def test_same_call_same_bits_on_any_stream_and_in_graphs(K, N):
    import torch
    import paper_2407_20496_amd as hinm
    gen = torch.Generator(device=DEV)
    gen.manual_seed(6)
    ld = N if N == 1 else (N + 7) // 8 * 8
    x, du, u, dx = (torch.randn(K, ld, device=DEV, generator=gen).bfloat16() for _ in range(4))
    w, b, dw, db = (torch.randn(K, device=DEV, generator=gen) for _ in range(4))
    mean, rstd = torch.empty(N, device=DEV), torch.empty(N, device=DEV)
    ws = workspace(max(hinm.hinm_layer_norm_workspace(K, N), hinm.hinm_layer_norm_grad_workspace(K, N)))

    def step(stream=None):
        hinm.hinm_layer_norm(K, N, "bf16", 1e-5, x, ld, w, b, u, ld, mean, rstd, *ws, stream=stream)
        hinm.hinm_layer_norm_grad(K, N, "bf16", x, ld, w, mean, rstd, du, ld, None, dx, dw, db, *ws, stream=stream)

    outputs = lambda: [t[:, :N].clone() if t.dim() == 2 else t.clone() for t in (u, mean, rstd, dx, dw, db)]
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
        for t in (u, mean, rstd, dx, dw, db):
            t.fill_(7)
        ws[0].fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outputs(), want))


def test_offsets_beyond_32_bits():
    import torch
    import paper_2407_20496_amd as hinm
    rng = np.random.default_rng(2)
    K, N, pitch = 1100, 70, 1 << 21
    x = _stream_values(rng, K, N, "bf16")
    whole = torch.empty(K * pitch, dtype=torch.bfloat16, device=DEV)
    view = whole.as_strided((K, N), (pitch, 1))
    view.copy_(torch.as_tensor(x, device=DEV).bfloat16())
    mean, rstd = torch.empty(N, device=DEV), torch.empty(N, device=DEV)
    u = result(K, N, "bf16")
    hinm.hinm_layer_norm(K, N, "bf16", 1e-5, whole, pitch, None, None, u.data, u.ld, mean, rstd,
                         *workspace(hinm.hinm_layer_norm_workspace(K, N)))
    got = (u.f64(), mean.double().cpu().numpy(), rstd.double().cpu().numpy())
    _check_forward(got, x, None, None, 1e-5, "bf16")
