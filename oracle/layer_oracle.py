"""fp64 CPU statement of the steps around the attention: rotary positions of q and k with their RMS norm, and the norms
before and after a block with modulation, gate and residual; forward and backward, written from the formulas.

numpy only; imports nothing of the library.  Beside each result stands `mag`, the sum of the absolute values of the terms it is
made of: what an error of fp32 arithmetic is measured against.
"""
import numpy as np


# ---- rotary positions ------------------------------------------------------------------------------------------------
def grid_positions(N, grid, origin=(0, 0, 0)):
    """int64 [N, 3]: tokens past the grid are at 0."""
    T, Y, X = grid
    pos = np.zeros((N, 3), dtype=np.int64)
    for n in range(min(N, T * Y * X)):
        pos[n] = (origin[0] + n // (Y * X), origin[1] + n // X % Y, origin[2] + n % X)
    return pos


def frequencies(axis_pairs, d, theta):
    f = np.zeros(d // 2)
    j = 0
    for n in axis_pairs:
        for i in range(n):
            f[j] = theta ** (-i / n)
            j += 1
    return f


def _angles(pos, freq, axis_pairs):
    """pos [B or 1, N, 3] -> [B or 1, 1, N, d / 2]"""
    axis = np.repeat(np.arange(3), axis_pairs)
    a = np.zeros(pos.shape[:2] + (freq.size,))
    a[..., :axis.size] = pos.astype(np.float64)[..., axis] * freq[:axis.size]
    return a[:, None]


def _split(x, halves):
    h = x.shape[-1] // 2
    return (x[..., :h], x[..., h:]) if halves else (x[..., 0::2], x[..., 1::2])


def _join(a, b, halves):
    if halves:
        return np.concatenate([a, b], -1)
    out = np.empty(a.shape[:-1] + (2 * a.shape[-1],))
    out[..., 0::2], out[..., 1::2] = a, b
    return out


def _turn(x, angle, halves):
    a, b = _split(x, halves)
    c, s = np.cos(angle), np.sin(angle)
    return _join(a * c - b * s, a * s + b * c, halves)


def _pair_mag(x, halves):
    a, b = _split(np.abs(x), halves)
    return _join(a + b, a + b, halves)


def _rms(x, norm, eps):
    """x [B, H, N, d] -> what it is multiplied with"""
    axes = (3,) if norm == "head" else (1, 3)
    return 1.0 / np.sqrt((x * x).mean(axes, keepdims=True) + eps)


def _wide(w, norm):
    """[d] or [H, d] as it meets [B, H, N, d]"""
    return 1.0 if w is None else w[:, None, :] if norm == "token" else w


def rope_forward(x, pos, freq, axis_pairs, halves=False, norm="none", w=None, eps=1e-6):
    """x [B, H, N, d], pos [B or 1, N, 3] -> (y, mag)"""
    m = x if norm == "none" else x * _rms(x, norm, eps) * _wide(w, norm)
    return _turn(m, _angles(pos, freq, axis_pairs), halves), _pair_mag(m, halves)


def rope_backward(x, dy, pos, freq, axis_pairs, halves=False, norm="none", w=None, eps=1e-6):
    """-> dict dx, dw (None without a norm) and their mag"""
    g = _turn(dy, -_angles(pos, freq, axis_pairs), halves)
    gm = _pair_mag(dy, halves)
    if norm == "none":
        return {"dx": g, "dx_mag": gm, "dw": None, "dw_mag": None}
    r = _rms(x, norm, eps)
    n, wide = x * r, _wide(w, norm)
    axes, over = ((3,), (0, 1, 2)) if norm == "head" else ((1, 3), (0, 2))
    t, tm = g * wide, gm * np.abs(wide)
    return {"dx": r * (t - n * (t * n).mean(axes, keepdims=True)),
            "dx_mag": r * (tm + np.abs(n) * (tm * np.abs(n)).mean(axes, keepdims=True)),
            "dw": (g * n).sum(over), "dw_mag": (gm * np.abs(n)).sum(over)}


# ---- norms around a block --------------------------------------------------------------------------------------------
def _norm(v, kind, eps):
    """v [B, N, C] -> (normalised, its mag, what it was multiplied with)"""
    if kind == "none":
        return v, np.abs(v), np.ones(v.shape[:-1] + (1,))
    mu = v.mean(-1, keepdims=True) if kind == "layer" else 0.0
    c = v - mu
    r = 1.0 / np.sqrt((c * c).mean(-1, keepdims=True) + eps)
    mag = np.abs(c) + (np.abs(v).mean(-1, keepdims=True) if kind == "layer" else 0.0)
    return c * r, mag * r, r


def _mod(m, layout, absent):
    """gate, scale or shift as it meets [B, N, C]"""
    return absent if m is None else m[:, None] if layout == "batch" else m


def _one(w):
    return 1.0 if w is None else w


def residual(x, y, kind, rho=1.0, gate=None, w=None, layout="batch", eps=1e-6):
    """x' = rho x + gate norm(y) w -> (x', mag)"""
    n, nm, _ = _norm(y, kind, eps)
    g = _mod(gate, layout, 1.0) * _one(w)
    return rho * x + g * n, np.abs(rho * x) + np.abs(g) * nm


def before(x, kind, w=None, scale=None, shift=None, layout="batch", eps=1e-6):
    """h = norm(x) w (1 + scale) + shift -> (h, mag)"""
    n, nm, _ = _norm(x, kind, eps)
    s = _mod(scale, layout, 0.0)
    a, am = _one(w) * (1.0 + s), np.abs(_one(w)) * (1.0 + np.abs(s))
    b = _mod(shift, layout, 0.0)
    return n * a + b, nm * am + np.abs(b)


def _norm_back(kind, n, nm, r, t, tm):
    if kind == "none":
        return t, tm
    dx, mag = t - n * (t * n).mean(-1, keepdims=True), tm + nm * (tm * nm).mean(-1, keepdims=True)
    if kind == "layer":
        dx, mag = dx - t.mean(-1, keepdims=True), mag + tm.mean(-1, keepdims=True)
    return dx * r, mag * r


def _mod_sum(terms, layout):
    return terms if layout == "token" else terms.sum(1) if layout == "batch" else terms.sum((0, 1))


def norm_backward(x, y, dh, dx_out, norm_in, norm_out, rho=1.0, gate=None, out_weight=None, in_weight=None, scale=None,
                  layout="batch", eps=1e-6):
    """The gradients of both steps: dict name -> (value, mag).  y, dh, dx_out may be None."""
    out = {}
    like = x if x is not None else y
    u = np.zeros_like(like) if dx_out is None else dx_out
    um = np.abs(u)
    if dh is not None:
        n, nm, r = _norm(x, norm_in, eps)
        s = _mod(scale, layout, 0.0)
        w = _one(in_weight)
        out["dshift"] = _mod_sum(dh, layout), _mod_sum(np.abs(dh), layout)
        out["dscale"] = _mod_sum(dh * n * w, layout), _mod_sum(np.abs(dh) * nm * np.abs(w), layout)
        one = np.ones_like(dh)
        out["din_weight"] = (dh * n * (1.0 + s)).sum((0, 1)), (np.abs(dh) * nm * (1.0 + np.abs(s)) * one).sum((0, 1))
        t, tm = dh * (w * (1.0 + s)), np.abs(dh) * np.abs(w) * (1.0 + np.abs(s))
        d, dm = _norm_back(norm_in, n, nm, r, t, tm)
        u, um = u + d, um + dm
    if y is not None:
        n, nm, r = _norm(y, norm_out, eps)
        w, g = _one(out_weight), _mod(gate, layout, 1.0)
        out["dgate"] = _mod_sum(u * n * w, layout), _mod_sum(um * nm * np.abs(w), layout)
        out["dout_weight"] = (u * n * g).sum((0, 1)), (um * nm * np.abs(g)).sum((0, 1))
        out["dy"] = _norm_back(norm_out, n, nm, r, u * (w * g), um * np.abs(w * g))
        u, um = rho * u, abs(rho) * um
    out["dx"] = u, um
    return out
