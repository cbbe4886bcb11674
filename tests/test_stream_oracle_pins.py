"""stream_oracle.py against library routines, automatic differentiation, differences and hand-worked cases (CPU)."""
import math

import numpy as np
import pytest
import torch

import stream_oracle as S


def sizes(rng, lens_q, lens_k, H, Hkv, d):
    q, k, v, g = (rng.normal(size=(sum(n), h, d)) for n, h in ((lens_q, H), (lens_k, Hkv), (lens_k, Hkv), (lens_q, H)))
    cut = lambda n: [0] + list(np.cumsum(n))  # noqa: E731
    return q, k, v, g, cut(lens_q), cut(lens_k)


def by_torch(q, k, v, qs, ks, causal, scale):
    out = []
    group = q.shape[1] // k.shape[1]
    for a, b, c, e in zip(qs, qs[1:], ks, ks[1:]):
        t = scale * torch.einsum("ihc,jhc->hij", q[a:b], k[c:e].repeat_interleave(group, 1))
        if causal:
            i, j = torch.arange(b - a)[:, None], torch.arange(e - c)[None]
            t = t.masked_fill(j > i + (e - c) - (b - a), -math.inf)
        w = torch.softmax(t, -1)
        w = torch.where(torch.isnan(w), 0.0, w)
        out.append(torch.einsum("hij,jhc->ihc", w, v[c:e].repeat_interleave(group, 1)))
    return torch.cat(out)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("lens", [([3, 1, 5], [3, 1, 5]), ([2, 4], [7, 4]), ([6, 3], [2, 3])])
def test_forward_and_gradients(causal, lens):
    rng = np.random.default_rng(1)
    q, k, v, g, qs, ks = sizes(rng, *lens, 4, 2, 8)
    scale = 0.3
    r = S.packed_forward(q, k, v, qs, ks, causal, scale)
    tq, tk, tv = (torch.from_numpy(x).requires_grad_() for x in (q, k, v))
    out = by_torch(tq, tk, tv, qs, ks, causal, scale)
    np.testing.assert_allclose(r["out"], out.detach().numpy(), atol=1e-13)
    b = S.packed_backward(q, k, v, qs, ks, causal, scale, r["out"], r["lse"], g)
    eps = 1e-6                                        # differences of the oracle's own forward pass
    for name, x in (("dq", q), ("dk", k), ("dv", v)):
        for at in [tuple(rng.integers(0, n) for n in x.shape) for _ in range(5)]:
            keep, f = x[at], []
            for s in (1, -1):
                x[at] = keep + s * eps
                f.append((S.packed_forward(q, k, v, qs, ks, causal, scale)["out"] * g).sum())
            x[at] = keep
            assert abs((f[0] - f[1]) / (2 * eps) - b[name][at]) < 1e-7, (name, at)
    if not (causal and lens[0] == [6, 3]):            # rows without a key: the library's softmax has no gradient there
        for name, want in zip(("dq", "dk", "dv"), torch.autograd.grad(out, (tq, tk, tv), torch.from_numpy(g))):
            np.testing.assert_allclose(b[name], want.numpy(), atol=1e-12, err_msg=name)


def test_empty_rows_and_sequences():
    rng = np.random.default_rng(2)
    q, k, v, g, qs, ks = sizes(rng, [3, 2, 2], [1, 0, 2], 2, 1, 4)
    r = S.packed_forward(q, k, v, qs, ks, True, 1.0)
    assert np.all(r["out"][[0, 1, 3, 4]] == 0) and np.all(r["lse"][:, [0, 1, 3, 4]] == -np.inf)
    np.testing.assert_array_equal(r["out"][2], np.repeat(v[0], 2, 0))      # one key: its value
    assert S.reads(3, 1, True).tolist() == [[False], [False], [True]]
    assert S.reads(2, 4, True).tolist() == [[True] * 3 + [False], [True] * 4]
    b = S.packed_backward(q, k, v, qs, ks, True, 1.0, r["out"], r["lse"], g)
    assert np.all(b["dq"][[0, 1, 3, 4]] == 0)
    assert S.bounds([0, 5, 3, 99], 7) == [(0, 5), (5, 0), (3, 4)]


def test_codes():
    x = np.array([[448.0, -224.0, 1.0, 0.0], [0.0, 0, 0, 0], [2.0 ** -101, 0, 0, 0], [np.inf, 1, 0, 0], [np.nan, 1, 0, 0]], dtype=np.float32)
    c, s = S.code_rows(x, "fp8")
    np.testing.assert_array_equal(c[:3], [[448, -224, 1, 0], [0] * 4, [0] * 4])
    assert s[0] == 1 and s[1] == 1 and s[2] == 1 and np.isnan(s[3]) and np.isnan(s[4]) and not c[3:].any()
    c, s = S.code_rows(np.array([[254.0, -3.0, 1.0, 5.0]], dtype=np.float32), "int8")
    np.testing.assert_array_equal(c, [[127, -2, 0, 2]])            # -1.5, 0.5, 2.5: ties to even
    assert s[0] == 2


def test_places():
    table = np.array([[3, 0], [9, -1]])
    assert S.place(0, 17, table, 16, 4) == (0, 1) and S.place(0, 32, table, 16, 4) is None and S.place(0, -1, table, 16, 4) is None
    assert S.place(1, 0, table, 16, 4) is None and S.place(1, 20, table, 16, 4) is None
    assert list(S.rows_of([1, 3, 3, 4], [5, 0, 2], 6, 3)) == [(1, 0, 5), (2, 0, 6), (3, 2, 2)]
    assert list(S.rows_of(None, None, 2, 5)) == [(0, 0, 0), (1, 1, 0)]
