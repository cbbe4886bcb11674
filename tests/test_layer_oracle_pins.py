"""The fp64 statement of the steps around the attention against what it must be: hand-worked values, invariants, and its
gradients against differences.  CPU only."""
import numpy as np
import pytest

import layer_oracle as L


def rng():
    return np.random.default_rng(7)


@pytest.mark.parametrize("halves", [False, True])
def test_rotation_of_a_known_angle(halves):
    # one head of 64 channels, axis 1 alone with frequency pi / 2 per row: a quarter turn at row 1
    d = 64
    x = np.zeros((1, 1, 2, d))
    x[0, 0, :, 0] = 3.0                                   # first channel of pair 0 in either order
    pos = np.array([[[5, 0, 9], [5, 1, 9]]])
    y, _ = L.rope_forward(x, pos, np.full(32, np.pi / 2), (0, 32, 0), halves)
    other = 32 if halves else 1
    assert y[0, 0, 0, 0] == 3.0 and abs(y[0, 0, 1, other] - 3.0) < 1e-15 and abs(y[0, 0, 1, 0]) < 1e-15
    assert np.count_nonzero(np.abs(y) > 1e-12) == 2


@pytest.mark.parametrize("halves", [False, True])
def test_scores_depend_on_differences_of_positions_only(halves):
    g, d = rng(), 128
    q, k = (g.normal(size=(1, 1, 1, d)) for _ in range(2))
    f = L.frequencies((22, 21, 21), d, 10000.0)
    score = lambda a, b: float((L.rope_forward(q, np.array([[a]]), f, (22, 21, 21), halves)[0] *      # noqa: E731
                                L.rope_forward(k, np.array([[b]]), f, (22, 21, 21), halves)[0]).sum())
    assert abs(score((3, 7, 11), (1, 2, 5)) - score((13, 27, 41), (11, 22, 35))) < 1e-11


def test_frequencies_and_grid():
    f = L.frequencies((2, 0, 1), 64, 100.0)
    assert f[0] == 1.0 and abs(f[1] - 0.1) < 1e-15 and f[2] == 1.0 and np.all(f[3:] == 0.0)
    p = L.grid_positions(8, (1, 2, 3), (10, 20, 30))
    assert p[4].tolist() == [10, 21, 31] and p[6:].tolist() == [[0, 0, 0]] * 2


def test_norms_of_a_known_row():
    v = np.array([[[1.0, -1.0, 3.0, 1.0]]])
    n, _, r = L._norm(v, "layer", 0.0)
    assert np.allclose(n, (v - 1.0) / np.sqrt(2.0)) and np.allclose(r, 1 / np.sqrt(2.0))
    n, _, r = L._norm(v, "rms", 0.0)
    assert np.allclose(n, v / np.sqrt(3.0))
    h, _ = L.before(v, "none", scale=np.full((1, 4), 0.5), shift=np.full((1, 4), 2.0))
    assert np.allclose(h, 1.5 * v + 2.0)
    x, _ = L.residual(v, v, "none", rho=2.0, gate=np.full((1, 4), -1.0))
    assert np.allclose(x, v)


def difference(f, x, at, step=1e-5):
    a, b = x.copy(), x.copy()
    a[at] += step
    b[at] -= step
    return (f(a) - f(b)) / (2 * step)


@pytest.mark.parametrize("norm", ["none", "head", "token"])
@pytest.mark.parametrize("halves", [False, True])
def test_rope_gradients_against_differences(norm, halves):
    g, B, H, N, d = rng(), 2, 3, 4, 64
    x, dy = g.normal(size=(B, H, N, d)), g.normal(size=(B, H, N, d))
    w = None if norm == "none" else g.normal(size=(d,) if norm == "head" else (H, d))
    pos, f = g.integers(-50, 50, size=(B, N, 3)), L.frequencies((5, 9, 12), d, 50.0)
    args = dict(halves=halves, norm=norm, eps=0.3)
    got = L.rope_backward(x, dy, pos, f, (5, 9, 12), w=w, **args)
    loss = lambda x_, w_: float((L.rope_forward(x_, pos, f, (5, 9, 12), w=w_, **args)[0] * dy).sum())       # noqa: E731
    for _ in range(12):
        at = tuple(int(g.integers(n)) for n in x.shape)
        assert abs(difference(lambda t: loss(t, w), x, at) - got["dx"][at]) < 1e-7
        if w is not None:
            at = tuple(int(g.integers(n)) for n in w.shape)
            assert abs(difference(lambda t: loss(x, t), w, at) - got["dw"][at]) < 1e-7


@pytest.mark.parametrize("layout", ["batch", "token", "shared"])
@pytest.mark.parametrize("kinds", [("rms", "rms"), ("layer", "none"), ("none", "layer"), ("layer", "rms")])
def test_norm_gradients_against_differences(layout, kinds):
    g, B, N, C = rng(), 2, 3, 16
    p = {"x": g.normal(size=(B, N, C)) + 0.5, "y": g.normal(size=(B, N, C)), "wo": g.normal(size=C), "wi": g.normal(size=C)}
    lead = {"batch": (B, C), "token": (B, N, C), "shared": (C,)}[layout]
    for k in ("gate", "scale", "shift"):
        p[k] = g.normal(size=lead)
    dh, dx_out, rho, eps = g.normal(size=(B, N, C)), g.normal(size=(B, N, C)), 0.7, 0.2

    def loss(**kw):
        q = dict(p, **kw)
        x1, _ = L.residual(q["x"], q["y"], kinds[1], rho, q["gate"], q["wo"], layout, eps)
        h, _ = L.before(x1, kinds[0], q["wi"], q["scale"], q["shift"], layout, eps)
        return float((h * dh).sum() + (x1 * dx_out).sum())

    x1, _ = L.residual(p["x"], p["y"], kinds[1], rho, p["gate"], p["wo"], layout, eps)
    got = L.norm_backward(x1, p["y"], dh, dx_out, kinds[0], kinds[1], rho, p["gate"], p["wo"], p["wi"], p["scale"], layout, eps)
    for name, key in (("x", "dx"), ("y", "dy"), ("gate", "dgate"), ("scale", "dscale"), ("shift", "dshift"), ("wo", "dout_weight"),
                      ("wi", "din_weight")):
        for _ in range(6):
            at = tuple(int(g.integers(n)) for n in p[name].shape)
            assert abs(difference(lambda t: loss(**{name: t}), p[name], at) - got[key][0][at]) < 1e-6, name
        assert np.all(got[key][1] >= np.abs(got[key][0]) - 1e-12), name
