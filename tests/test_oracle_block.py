"""Pins of the oracle of the 4-bit form and of a block's norms (CPU only)."""
import numpy as np
import pytest

from oracle import block_oracle as orc


def _nearest(a):
    """Code of a / scale by search over the whole list: nearest value, ties to the even place."""
    best = min(range(8), key=lambda i: (abs(abs(a) - orc.LEVELS[i]), i % 2))
    return best | (8 if np.signbit(a) else 0)


def test_rounding_to_codes():
    rng = np.random.default_rng(0)
    grid = np.concatenate([np.arange(-8, 8.001, 0.125), rng.uniform(-7.9, 7.9, 60)])
    X = np.zeros((grid.size, 32))
    X[:, 0] = 4.0                # fixes the scale at one
    X[:, 1] = np.where(np.abs(grid) < 8, grid, np.sign(grid) * 7.875)
    codes, scales = orc.quantize_rows(X)
    assert (scales[:, 0] == 127).all()
    assert [int(c) for c in codes[:, 0] >> 4] == [_nearest(v) for v in X[:, 1]]


def test_scales_and_their_places():
    X = np.zeros((1, 1024))
    for j in range(32):
        X[0, 32 * j + j] = 2.0 ** (j - 10) * 1.5
    codes, scales = orc.quantize_rows(X)
    for j in range(32):
        byte = scales[0, 16 * (j // 16) + 4 * (j % 4) + (j % 16) // 4]
        assert byte == j - 10 - 2 + 127
    assert np.array_equal(orc.values(codes, scales, 1024), X)
    assert sorted(orc.scale_place(j) for j in range(32)) == list(range(32))


def test_order_in_memory():
    """Every byte where include/hinm.h says it is."""
    rng = np.random.default_rng(2)
    rows, length = 37, 700
    c, s = orc.quantize_rows(rng.standard_normal((rows, length)))
    mc, ms = orc.to_memory(c, s, 9)
    mc, ms = mc.reshape(3, 2, 4, 2, 32, 16), ms.reshape(2, 2, 32, 16)
    for r in (0, 5, 31, 32, 36):
        for k in (0, 31, 32, 64, 100, 129, 200, 255, 256, 511, 600, 699):
            p, j = k % 256 // 32, k % 512 // 32
            assert mc[k // 256, r // 32, 2 * (p // 4) + p % 2, p // 2 % 2, r % 32, k % 32 // 2] == c[r, k // 2]
            assert ms[k // 512, r // 32, r % 32, 4 * (j % 4) + j // 4] == s[r, orc.scale_place(k // 32)]
    assert (mc[:, 1, :, :, 5:] == 9).all() and (ms[:, 1, 5:] == 9).all()
    back = orc.from_memory(mc.reshape(-1), ms.reshape(-1), rows)
    assert np.array_equal(back[0][:rows], c) and np.array_equal(back[1][:rows], s)


def test_special_blocks():
    X = np.zeros((1, 160))
    X[0, 32] = np.inf
    X[0, 70] = np.nan
    X[0, 96] = 2.0 ** -133        # below every scale: the smallest one is kept
    codes, scales = orc.quantize_rows(X)
    assert [int(scales[0, orc.scale_place(j)]) for j in range(6)] == [0, 255, 255, 0, 0, 127]
    v = orc.values(codes, scales, 160)
    assert np.isnan(v[0, 32:96]).all() and (v[0, :32] == 0).all() and (v[0, 96:] == 0).all()


def test_values_are_near_and_kept_by_a_second_pass():
    X = np.random.default_rng(1).standard_normal((9, 333))
    c, s = orc.quantize_rows(X)
    V = orc.values(c, s, 333)
    e = np.stack([s[:, orc.scale_place(j)] for j in np.arange(333) // 32], axis=1).astype(np.float64)
    unit = 2.0 ** (e - 127)
    assert (np.abs(V - X) <= np.where(np.abs(X) / unit > 6, 2, 1) * unit).all()
    again = orc.values(*orc.quantize_rows(V), 333)
    assert np.array_equal(again, V)


FORMS = [dict(post=p, gate=g, token=t, pre=n, block=b) for p in (0, 1) for g in (0, 1) for t in (0, 1) for n in (0, 1)
         for b in (0, 1) if (b or not (p or g or t)) and (b or n)]


def draw(K, N, form, seed):
    rng = np.random.default_rng(seed)
    on = lambda flag, v: v if flag else None
    return {"x": rng.standard_normal((K, N)), "y": on(form["block"], rng.standard_normal((K, N))),
            "w_post": on(form["post"], 1 + 0.3 * rng.standard_normal(K)), "gate": on(form["gate"], rng.standard_normal(K)),
            "token_gate": on(form["token"], rng.standard_normal(N)), "w_pre": on(form["pre"], 1 + 0.3 * rng.standard_normal(K))}


@pytest.mark.parametrize("form", FORMS, ids=lambda f: "".join(k for k, v in f.items() if v))
def test_gradients_against_differences(form):
    """Central differences of the forward formulas in binary64: error of the order of step^2 and of 1e-16 / step."""
    K, N, scale, eps = 5, 3, 0.7, 1e-3
    a = draw(K, N, form, 3)
    rng = np.random.default_rng(4)
    dh = rng.standard_normal((K, N))
    du = rng.standard_normal((K, N)) if form["pre"] else None

    def loss(b):
        r = orc.block_norm(b["x"], b["y"], b["w_post"], b["gate"], b["token_gate"], b["w_pre"], scale, eps)
        return (r["h"] * dh).sum() + (0 if du is None else (r["u"] * du).sum())
    r = orc.block_norm(a["x"], a["y"], a["w_post"], a["gate"], a["token_gate"], a["w_pre"], scale, eps)
    got = orc.block_norm_grad(r["h"], a["y"], a["w_post"], a["gate"], a["token_gate"], a["w_pre"], r["rstd_y"], r["rstd_h"],
                              dh, du, scale)
    names = {"dx": "x", "dy": "y", "dw_post": "w_post", "dgate": "gate", "dtoken_gate": "token_gate", "dw_pre": "w_pre"}
    assert set(got) == {n for n, v in names.items() if a[v] is not None}
    step = 1e-5
    for name, (value, size) in got.items():
        v = a[names[name]]
        for i in np.ndindex(v.shape):
            moved = []
            for sign in (1, -1):
                b = {k: None if t is None else t.copy() for k, t in a.items()}
                b[names[name]][i] += sign * step
                moved.append(loss(b))
            assert abs((moved[0] - moved[1]) / (2 * step) - value[i]) < 1e-7 * (1 + size[i]), (name, i)
