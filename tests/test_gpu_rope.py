"""sla2_rope_forward and sla2_rope_backward through the C ABI against the fp64 statement of the same."""
import numpy as np
import pytest

import layer_oracle as L
from layer_helpers import GUARD, TRIG_UNITS, close, f64, guards_ok, heads_like, sum_units

pytestmark = pytest.mark.gpu

NORMS = ["none", "head", "token"]


def types(torch, name):
    return torch.bfloat16 if name == "bf16" else torch.float32


class Case:
    """Inputs of one call, and the call."""

    def __init__(self, B, H, N, d, dtype="bf16", halves=False, norm="token", layout="packed", out_layout="tokens", axes=None, grid=None,
                 origin=(0, 0, 0), per_batch=1, positions=None, weights=True, eps=1e-5, seed=0):
        import torch
        from paper_2602_12675_amd import api
        self.torch, self.api = torch, api
        self.B, self.H, self.N, self.d, self.norm, self.halves, self.eps = B, H, N, d, norm, halves, eps
        self.layout, self.out_layout, self.dtype = layout, out_layout, types(torch, dtype)
        gen = self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.axes = axes or (d // 2 - 2 * (d // 6), d // 6, d // 6)
        (self.q, self.k), self.ist, self.ibufs = heads_like(torch, B, H, N, d, layout, self.dtype, gen)
        _, self.ost, _ = heads_like(torch, B, H, N, d, out_layout, self.dtype)
        shape = (H, d) if norm == "token" else (d,)
        self.w = [1 + 0.3 * torch.randn(shape, generator=gen, device="cuda") for _ in range(2)] if norm != "none" and weights else [None] * 2
        self.grid = grid
        if grid is None:
            if positions is None:
                positions = torch.randint(-3000, 3000, (B if per_batch else 1, N, 3), generator=gen, device="cuda")
            self.pos = positions.int().contiguous()
            self.pos64 = f64(self.pos).astype(np.int64)
        else:
            self.pos, self.pos64 = None, L.grid_positions(N, grid, origin)[None]
        self.p = api.make_rope_params(B, H, N, d, self.axes, grid=grid or (0, 0, 0), origin=origin,
                                      dtype=api.SLA2_BF16 if dtype == "bf16" else api.SLA2_F32, pairing=int(halves),
                                      norm=NORMS.index(norm), eps=eps, positions_per_batch=per_batch, in_stride=self.ist,
                                      out_stride=self.ost)
        self.freq = api.sla2_rope_frequencies(self.p).cuda()
        self.units = TRIG_UNITS if dtype == "bf16" else 64

    def forward(self, **kw):
        (qo, ko), _, bufs = heads_like(self.torch, self.B, self.H, self.N, self.d, self.out_layout, self.dtype)
        self.api.sla2_rope_forward(self.p, self.q, self.k, self.freq, qo, ko, q_weight=self.w[0], k_weight=self.w[1], positions=self.pos, **kw)
        return qo, ko, bufs

    def reference(self, x, w):
        return L.rope_forward(f64(x), self.pos64, f64(self.freq), self.axes, self.halves, self.norm, None if w is None else f64(w), self.eps)

    def check_forward(self):
        qo, ko, bufs = self.forward()
        self.torch.cuda.synchronize()
        for x, w, got, name in ((self.q, self.w[0], qo, "q"), (self.k, self.w[1], ko, "k")):
            close(got, *self.reference(x, w), self.dtype, self.units, name)
        guards_ok(self.out_layout, bufs)
        return qo, ko

    def check_backward(self):
        torch = self.torch
        (gq, gk), _, _ = heads_like(torch, self.B, self.H, self.N, self.d, self.out_layout, self.dtype, self.gen)
        (dq, dk), _, bufs = heads_like(torch, self.B, self.H, self.N, self.d, self.layout, self.dtype)
        dw = [torch.full((self.H, self.d) if self.norm == "token" else (self.d,), GUARD, device="cuda") if self.norm != "none" else None
              for _ in range(2)]
        ws = torch.empty(self.api.sla2_rope_workspace_bytes(self.p), dtype=torch.uint8, device="cuda").fill_(255)
        self.api.sla2_rope_backward(self.p, self.q, self.k, self.freq, gq, gk, dq, dk, q_weight=self.w[0], k_weight=self.w[1],
                                    dq_weight=dw[0], dk_weight=dw[1], positions=self.pos, workspace=ws)
        torch.cuda.synchronize()
        for x, g, w, dx, dwi, name in ((self.q, gq, self.w[0], dq, dw[0], "q"), (self.k, gk, self.w[1], dk, dw[1], "k")):
            ref = L.rope_backward(f64(x), f64(g), self.pos64, f64(self.freq), self.axes, self.halves, self.norm,
                                  None if w is None else f64(w), self.eps)
            close(dx, ref["dx"], ref["dx_mag"], self.dtype, self.units, "d" + name)
            if dwi is not None:
                close(dwi, ref["dw"], ref["dw_mag"], torch.float32, self.units + sum_units(self.N), "d%s weight" % name)
        guards_ok(self.layout, bufs)
        return gq, gk, dq, dk, dw


SIZES = [(1, 1, 1, 64), (1, 1, 1, 128), (2, 1, 5, 64), (1, 3, 67, 64), (2, 5, 33, 128), (1, 12, 40, 128), (2, 16, 17, 64), (3, 20, 31, 64),
         (1, 9, 21, 128), (1, 40, 9, 128), (1, 64, 5, 128), (5, 2, 700, 64)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("norm", NORMS)
@pytest.mark.parametrize("halves", [False, True], ids=["pairs", "halves"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_forward_and_backward(size, halves, norm, dtype):
    c = Case(*size, dtype=dtype, halves=halves, norm=norm, seed=sum(size))
    c.check_forward()
    c.check_backward()


@pytest.mark.parametrize("layout,out_layout", [("heads", "heads"), ("heads", "padded"), ("padded", "heads"), ("tokens", "packed"),
                                               ("packed", "packed"), ("padded", "padded")])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_layouts(layout, out_layout, dtype):
    for norm in NORMS:
        c = Case(2, 6, 45, 64, dtype=dtype, norm=norm, halves=True, layout=layout, out_layout=out_layout, seed=3)
        c.check_forward()
        c.check_backward()


@pytest.mark.parametrize("H,d,norm", [(70, 128, "head"), (129, 64, "none"), (200, 64, "head"), (257, 128, "none")])
def test_more_heads_than_a_row_holds(H, d, norm):
    c = Case(1, H, 6, d, norm=norm, halves=(H % 2 == 0), seed=H)
    c.check_forward()
    c.check_backward()


@pytest.mark.parametrize("norm", NORMS)
def test_many_sequences_of_one_token(norm):
    c = Case(65535, 1, 1, 64, norm=norm, layout="tokens")
    c.check_forward()
    c.check_backward()


@pytest.mark.parametrize("H,N,d,norm", [(1, 127, 64, "token"), (1, 128, 64, "token"), (1, 129, 64, "head"), (1, 128, 64, "head"), (1, 64, 128, "head"),
                                        (3, 32, 64, "head"), (3, 33, 64, "token"), (12, 5, 128, "token"), (12, 6, 128, "head"),
                                        (64, 1, 128, "token"), (128, 2, 64, "head")])
@pytest.mark.parametrize("halves", [False, True])
def test_rows_of_one_workgroup(H, N, d, norm, halves):
    """As many rows as one workgroup takes side by side, whose sums need no second launch, and one more."""
    Case(1, H, N, d, norm=norm, halves=halves, dtype="f32" if halves else "bf16", seed=N).check_backward()


@pytest.mark.parametrize("axes", [(32, 0, 0), (0, 0, 32), (8, 12, 12), (0, 7, 3), (0, 0, 0), (1, 1, 1)])
@pytest.mark.parametrize("halves", [False, True])
def test_axes_and_channels_left_alone(axes, halves):
    """Pairs behind those of the axes are not rotated: bit for bit, without a norm."""
    c = Case(2, 3, 50, 64, dtype="f32", norm="none", halves=halves, axes=axes, seed=1)
    qo, _ = c.check_forward()
    n = sum(axes)
    idle = list(range(n, 32)) + list(range(32 + n, 64)) if halves else list(range(2 * n, 64))
    assert c.torch.equal(qo[..., idle], c.q[..., idle])
    c.check_backward()


@pytest.mark.parametrize("grid,N,origin", [((1, 64, 64), 4096, (0, 0, 0)), ((3, 5, 7), 105, (0, 0, 0)), ((3, 5, 7), 111, (20, 0, 0)),
                                           ((2, 3, 4), 24, (-5, 100000, 7)), ((1, 1, 1), 3, (9, 9, 9)), ((4, 9, 11), 200, (2147483644, 1, 2)),
                                           ((1, 1, 2147483647), 77, (0, 0, 0))])
def test_grid(grid, N, origin):
    c = Case(2, 2, N, 64, dtype="f32", norm="head", grid=grid, origin=origin, seed=N)
    c.check_forward()
    c.check_backward()


def test_grid_is_its_positions_and_tokens_past_it_are_not_rotated():
    import torch
    grid, N = (3, 4, 5), 66
    c = Case(2, 3, N, 128, norm="none", grid=grid, layout="tokens")
    p = Case(2, 3, N, 128, norm="none", positions=torch.from_numpy(L.grid_positions(N, grid)).cuda()[None], per_batch=0, layout="tokens")
    for a, b in zip(c.forward()[:2], p.forward()[:2]):
        assert torch.equal(a, b)
    qo = c.forward()[0]
    assert torch.equal(qo[:, :, 60:], c.q[:, :, 60:])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_far_positions(dtype):
    """Angles of 2^31 radians: exact to the 2^-53 of their own size (2.4e-7), the product's and the turn's, 3 of them: 12 units."""
    import torch
    far = torch.tensor([[2 ** 31 - 1, -2 ** 31, 2 ** 31 - 2], [-(2 ** 31) + 1, 2 ** 30 + 1, 123456789], [1, -1, 0], [0, 0, 0]])
    c = Case(1, 2, 4, 128, dtype=dtype, norm="none", positions=far[None].cuda(), per_batch=0)
    c.units += 12
    c.check_forward()
    c.check_backward()


def test_positions_shared_by_the_batch():
    c = Case(3, 2, 37, 64, per_batch=0, norm="head")
    assert c.pos.shape[0] == 1
    c.check_forward()
    c.check_backward()


@pytest.mark.parametrize("norm", NORMS)
def test_q_alone(norm):
    import torch
    c = Case(2, 3, 29, 64, norm=norm, layout="tokens")
    qo, ko, _ = c.forward()
    one = torch.full_like(qo, GUARD)
    st = one.stride()
    p = c.api.make_rope_params(2, 3, 29, 64, c.axes, norm=NORMS.index(norm), eps=c.eps, positions_per_batch=1, in_stride=c.ist,
                               out_stride=(st[0], st[1], st[2]))
    c.api.sla2_rope_forward(p, c.q, None, c.freq, one, None, q_weight=c.w[0], positions=c.pos)
    assert torch.equal(one, qo)
    g, dq, dk = torch.randn_like(qo), torch.empty_like(c.q), torch.empty_like(c.q)
    both = [torch.empty_like(c.w[0]) for _ in range(3)] if norm != "none" else [None] * 3
    ws = torch.empty(c.api.sla2_rope_workspace_bytes(c.p), dtype=torch.uint8, device="cuda")
    c.api.sla2_rope_backward(p, c.q, c.k, c.freq, g, g, dq, dk, q_weight=c.w[0], k_weight=c.w[1], dq_weight=both[0], dk_weight=both[1],
                             positions=c.pos, workspace=ws)
    dq1 = torch.empty_like(dq)
    c.api.sla2_rope_backward(p, c.q, None, c.freq, g, None, dq1, None, q_weight=c.w[0], dq_weight=both[2], positions=c.pos, workspace=ws)
    assert torch.equal(dq, dq1)
    if norm != "none":
        assert torch.equal(both[0], both[2])
    # without the gradients of the weights: no workspace, the same dq
    c.api.sla2_rope_backward(p, c.q, None, c.freq, g, None, dq1.fill_(GUARD), None, q_weight=c.w[0], positions=c.pos)
    assert torch.equal(dq, dq1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("norm", NORMS)
@pytest.mark.parametrize("H", [3, 12])
def test_in_place(norm, dtype, H):
    """q and k rotated where they lie in the packed projection, and back in the packed gradient: the bits of the other call, and v left."""
    import torch
    c = Case(2, H, 41, 128, dtype=dtype, norm=norm, layout="packed", out_layout="packed")
    want_q, want_k, _ = c.forward()
    gq, gk, dq, dk, dw = c.check_backward()
    x = c.ibufs[0].clone()
    q, k = (x[:, :, i].permute(0, 2, 1, 3) for i in range(2))
    c.api.sla2_rope_forward(c.p, q, k, c.freq, q, k, q_weight=c.w[0], k_weight=c.w[1], positions=c.pos)
    assert torch.equal(q, want_q) and torch.equal(k, want_k) and bool((x[:, :, 2] == GUARD).all())
    g = torch.full_like(x, GUARD)
    a, b = (g[:, :, i].permute(0, 2, 1, 3) for i in range(2))
    a.copy_(gq)
    b.copy_(gk)
    c.api.sla2_rope_backward(c.p, c.q, c.k, c.freq, a, b, a, b, q_weight=c.w[0], k_weight=c.w[1], positions=c.pos)
    assert torch.equal(a, dq) and torch.equal(b, dk) and bool((g[:, :, 2] == GUARD).all())
    if norm != "none":                                # over the saved inputs
        x = c.ibufs[0].clone()
        q, k = (x[:, :, i].permute(0, 2, 1, 3) for i in range(2))
        c.api.sla2_rope_backward(c.p, q, k, c.freq, gq, gk, q, k, q_weight=c.w[0], k_weight=c.w[1], positions=c.pos)
        assert torch.equal(q, dq) and torch.equal(k, dk)


def test_rotation_back_is_the_inverse():
    import torch
    c = Case(1, 4, 300, 128, dtype="f32", norm="none", layout="tokens")
    qo, ko, _ = c.forward()
    q, k = (torch.empty_like(qo) for _ in range(2))
    c.api.sla2_rope_backward(c.p, None, None, c.freq, qo, ko, q, k, positions=c.pos)
    torch.testing.assert_close(q, c.q, rtol=0, atol=64 * 2.0 ** -24 * 8)
    torch.testing.assert_close(k, c.k, rtol=0, atol=64 * 2.0 ** -24 * 8)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("norm", NORMS)
def test_what_is_not_finite_stays_in_its_row(norm, bad):
    import torch
    for H, d in ((1, 64), (3, 64), (12, 128)):
        c = Case(1, H, 50, d, norm=norm, layout="tokens")
        want_q, want_k, _ = c.forward()
        c.q[0, H - 1, 20, 3] = bad
        qo, ko, _ = c.forward()
        assert torch.equal(ko, want_k)
        keep = torch.ones(H, 50, dtype=torch.bool, device="cuda")
        if norm == "token":
            keep[:, 20] = False
        else:
            keep[H - 1, 20] = False
        assert torch.equal(qo[0][keep], want_q[0][keep])
        assert not bool(torch.isfinite(qo[0, H - 1, 20]).all())


def test_zero_rows():
    """All-zero tokens (padding) give zeros, and gradients of dy w / sqrt(eps)."""
    for norm in ("head", "token"):
        c = Case(2, 5, 19, 64, dtype="f32", norm=norm, layout="tokens", eps=1e-2)
        c.q[:, :, 3:9] = 0
        c.k[1] = 0
        qo, ko = c.check_forward()
        assert bool((qo[:, :, 3:9] == 0).all()) and bool((ko[1] == 0).all())
        c.check_backward()


def test_offsets_beyond_32_bits():
    import torch
    from paper_2602_12675_amd import api
    H, d, N, tok = 2, 64, 5, 1 << 30                   # five tokens 2^30 elements apart: 8 GB of bf16
    buf = torch.empty((N - 1) * tok + 2 * H * d, dtype=torch.bfloat16, device="cuda")
    at = lambda i: torch.as_strided(buf, (1, H, N, d), ((N - 1) * tok + 2 * H * d, d, tok, 1), i * H * d)      # noqa: E731
    q, k = at(0), at(1)
    q.copy_(torch.randn(q.shape, device="cuda"))
    k.copy_(torch.randn(q.shape, device="cuda"))
    st = ((N - 1) * tok + 2 * H * d, d, tok)
    pos = torch.randint(0, 99, (N, 3), device="cuda").int()
    far = api.make_rope_params(1, H, N, d, (10, 11, 11), norm=api.SLA2_ROPE_NORM_TOKEN, in_stride=st, out_stride=st)
    near = api.make_rope_params(1, H, N, d, (10, 11, 11), norm=api.SLA2_ROPE_NORM_TOKEN)
    freq = api.sla2_rope_frequencies(far).cuda()
    qc, kc = q.contiguous(), k.contiguous()
    qo, ko = torch.empty_like(qc), torch.empty_like(kc)
    api.sla2_rope_forward(near, qc, kc, freq, qo, ko, positions=pos)
    api.sla2_rope_forward(far, q, k, freq, q, k, positions=pos)
    assert torch.equal(q, qo) and torch.equal(k, ko)


def test_another_stream_and_a_captured_call():
    """On a side stream, then captured: every replay gives the eager bits."""
    import torch
    c = Case(2, 12, 500, 128, norm="token", layout="packed")
    gq, gk, dq, dk, dw = c.check_backward()
    want = [t.clone() for t in (*c.forward()[:2], dq, dk, *dw)]
    (qo, ko), _, _ = heads_like(torch, c.B, c.H, c.N, c.d, c.out_layout, c.dtype)
    (dq2, dk2), _, _ = heads_like(torch, c.B, c.H, c.N, c.d, c.layout, c.dtype)
    dw2 = [torch.empty_like(t) for t in dw]
    ws = torch.empty(c.api.sla2_rope_workspace_bytes(c.p), dtype=torch.uint8, device="cuda")
    got = [qo, ko, dq2, dk2, *dw2]

    def both(stream):
        c.api.sla2_rope_forward(c.p, c.q, c.k, c.freq, qo, ko, q_weight=c.w[0], k_weight=c.w[1], positions=c.pos, stream=stream)
        c.api.sla2_rope_backward(c.p, c.q, c.k, c.freq, gq, gk, dq2, dk2, q_weight=c.w[0], k_weight=c.w[1], dq_weight=dw2[0],
                                 dk_weight=dw2[1], positions=c.pos, workspace=ws, stream=stream)

    def check(what):
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b), what
            a.fill_(GUARD)
        ws.random_(0, 255)
        torch.cuda.synchronize()

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    both(side)
    check("side stream")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            both(side)
    torch.cuda.synchronize()
    for rep in range(3):
        graph.replay()
        check(rep)
