"""The attention part of a diffusion transformer's layer as it is used, forward and backward: norm and modulation, projection, norm and
rotation of q and k, sla2_forward, projection, gate and residual with the norm before the next block - and back.  Against the fp64
statements of the steps chained up, with the projections as plain matrix products; and captured into a graph."""
import numpy as np
import pytest

import layer_oracle as L
import sla2_oracle as O
from layer_helpers import f64

pytestmark = pytest.mark.gpu


class Layer:
    def __init__(self, B, grid, H, d, dtype, norm, extra=0, block_q=64, topk=0.2, seed=0):
        import torch
        from paper_2602_12675_amd import api
        self.torch, self.api = torch, api
        T, Y, X = grid
        self.B, self.N, self.H, self.d, self.C, self.bq, self.topk = B, T * Y * X + extra, H, d, H * d, block_q, topk
        N, C = self.N, self.C
        self.grid, self.norm = grid, norm
        f32 = dtype == "f32"
        self.th = torch.float32 if f32 else torch.bfloat16
        g = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda *s: torch.randn(s, generator=g, device="cuda")                                       # noqa: E731
        self.x = rand(B, N, C)                                               # residual stream in fp32
        self.e = 0.3 * rand(B, 6, C)                                         # modulation of this block and of the next one
        self.wqkv = (rand(C, 3 * C) / C ** 0.5).to(self.th)
        self.wo = (rand(C, C) / C ** 0.5).to(self.th)
        self.qw, self.kw = (1 + 0.2 * rand(*((H, d) if norm == "token" else (d,))) for _ in range(2))
        self.rw = rand(2, d, d) / d ** 0.5
        self.alpha = torch.rand((H,), generator=g, device="cuda")
        self.dx1, self.dh1 = rand(B, N, C), rand(B, N, C).to(self.th)
        st = (N * 3 * C, d, 3 * C)                                           # packed projection
        ost = (N * C, d, C)
        code = api.SLA2_F32 if f32 else api.SLA2_BF16
        self.np = api.make_norm_params(B, N, C, dtype_x=api.SLA2_F32, dtype_h=code, norm_in=api.SLA2_NORM_LAYER, mod_stride=(6 * C, 0))
        pairs = d // 2
        self.axes = (pairs - 2 * (pairs // 3), pairs // 3, pairs // 3)
        self.rp = api.make_rope_params(B, H, N, d, self.axes, grid=grid, dtype=code, norm={"head": 1, "token": 2}[norm], in_stride=st, out_stride=st)
        self.ap = api.make_params(B, H, N, d, block_q, 64, topk, dtype=code, flags=api.SLA2_FLAG_SAVE_FOR_BACKWARD, in_stride=st, out_stride=ost)
        self.freq = api.sla2_rope_frequencies(self.rp).cuda()
        self.aws = api.alloc_workspace(self.ap)
        self.ws = torch.empty(max(api.sla2_norm_workspace_bytes(self.np), api.sla2_rope_workspace_bytes(self.rp)), dtype=torch.uint8, device="cuda")
        self.idx = torch.empty((B, H, -(-N // block_q), api.sla2_num_selected(self.ap)), dtype=torch.int32, device="cuda")

    def slices(self, t):
        return [t[:, :, i] for i in range(3)]                                # [B, N, H, d]: q, k, v of a packed [B, N, 3, H, d]

    def run(self, stream=None):
        """One step; the results by name."""
        torch, api, e = self.torch, self.api, self.e
        B, N, H, d, C = self.B, self.N, self.H, self.d, self.C
        kw = dict(stream=stream)
        h = torch.empty((B, N, C), dtype=self.th, device="cuda")
        api.sla2_norm_forward(self.np, self.x, h, scale=e[:, 0], shift=e[:, 1], **kw)
        qkv = (h.view(B * N, C) @ self.wqkv).view(B, N, 3, H, d)
        turned = torch.empty_like(qkv)
        q, k, v = self.slices(qkv)
        tq, tk, _ = self.slices(turned)
        api.sla2_rope_forward(self.rp, q, k, self.freq, tq, tk, q_weight=self.qw, k_weight=self.kw, **kw)
        o = torch.empty((B, N, H, d), dtype=self.th, device="cuda")
        api.sla2_forward(self.ap, tq, tk, v, self.rw, self.alpha, o, block_idx=self.idx, workspace=self.aws, **kw)
        y = (o.view(B * N, C) @ self.wo).view(B, N, C)
        x1, h1 = torch.empty_like(self.x), torch.empty_like(h)
        api.sla2_norm_forward(self.np, self.x, h1, y=y, x_out=x1, gate=e[:, 2], scale=e[:, 3], shift=e[:, 4], **kw)
        # back
        de = torch.zeros_like(e)
        dx, dy = torch.empty_like(self.x), torch.empty_like(y)
        api.sla2_norm_backward(self.np, x1, self.dh1, self.dx1, dx, y=y, gate=e[:, 2], scale=e[:, 3], dy=dy, dgate=de[:, 2],
                               dscale=de[:, 3], dshift=de[:, 4], workspace=self.ws, **kw)
        do = (dy.view(B * N, C) @ self.wo.t()).view(B, N, H, d)
        dqkv = torch.empty_like(qkv)
        dq, dk, dv = self.slices(dqkv)
        dal = torch.empty_like(self.alpha)
        api.sla2_backward(self.ap, tq, tk, v, self.alpha, do, dq, dk, dv, dal, self.aws, **kw)
        dqw, dkw = torch.empty_like(self.qw), torch.empty_like(self.kw)
        api.sla2_rope_backward(self.rp, q, k, self.freq, dq, dk, dq, dk, q_weight=self.qw, k_weight=self.kw, dq_weight=dqw, dk_weight=dkw,
                               workspace=self.ws, **kw)
        dh = (dqkv.view(B * N, 3 * C) @ self.wqkv.t()).view(B, N, C)
        api.sla2_norm_backward(self.np, self.x, dh, dx, dx, scale=e[:, 0], dscale=de[:, 0], dshift=de[:, 1], workspace=self.ws, **kw)
        return {"x1": x1, "h1": h1, "dx": dx, "de": de[:, :5], "dqw": dqw, "dkw": dkw, "dalpha": dal}

    def reference(self):
        """The same in fp64, for the block lists of the run."""
        B, N, H, d, C = self.B, self.N, self.H, self.d, self.C
        x, e, wqkv, wo = f64(self.x), f64(self.e), f64(self.wqkv), f64(self.wo)
        pos, freq, idx, alpha = L.grid_positions(N, self.grid)[None], f64(self.freq), self.idx.cpu().numpy(), f64(self.alpha)
        args, rw = dict(norm=self.norm, eps=1e-6), f64(self.rw)
        h, _ = L.before(x, "layer", scale=e[:, 0], shift=e[:, 1])
        q, k, v = (h @ wqkv).reshape(B, N, 3, H, d).transpose(2, 0, 3, 1, 4)
        tq, tk = (L.rope_forward(t, pos, freq, self.axes, w=f64(w), **args)[0] for t, w in ((q, self.qw), (k, self.kw)))
        o = np.zeros((B, H, N, d))
        for b in range(B):
            for i in range(H):
                o[b, i] = O.forward_head(tq[b, i], tk[b, i], v[b, i], rw[0], rw[1], alpha[i], self.topk, self.bq, 64, sel=idx[b, i])["O"]
        y = o.transpose(0, 2, 1, 3).reshape(B, N, C) @ wo
        x1, _ = L.residual(x, y, "none", gate=e[:, 2])
        h1, _ = L.before(x1, "layer", scale=e[:, 3], shift=e[:, 4])
        g = L.norm_backward(x1, y, f64(self.dh1), f64(self.dx1), "layer", "none", gate=e[:, 2], scale=e[:, 3])
        do = (g["dy"][0] @ wo.T).reshape(B, N, H, d).transpose(0, 2, 1, 3)
        dq, dk, dv = (np.zeros((B, H, N, d)) for _ in range(3))
        dal = np.zeros(H)
        for b in range(B):
            for i in range(H):
                r = O.backward_head(tq[b, i], tk[b, i], v[b, i], idx[b, i], alpha[i], do[b, i], self.bq, 64)
                dq[b, i], dk[b, i], dv[b, i] = r["dQ"], r["dK"], r["dV"]
                dal[i] += r["dalpha"].sum()
        rq = L.rope_backward(q, dq, pos, freq, self.axes, w=f64(self.qw), **args)
        rk = L.rope_backward(k, dk, pos, freq, self.axes, w=f64(self.kw), **args)
        dqkv = np.stack([rq["dx"], rk["dx"], dv]).transpose(1, 3, 0, 2, 4).reshape(B, N, 3 * C)
        f = L.norm_backward(x, None, dqkv @ wqkv.T, g["dx"][0], "layer", "none", scale=e[:, 0])
        de = np.stack([f["dscale"][0], f["dshift"][0], g["dgate"][0], g["dscale"][0], g["dshift"][0]], 1)
        return {"x1": x1, "h1": h1, "dx": f["dx"][0], "de": de, "dqw": rq["dw"], "dkw": rk["dw"], "dalpha": dal}


# fp32: the attention's own bounds (2e-3 of values of order 1 in the forward pass) are far above its errors of about 1e-6, which the
# steps here carry on at most tenfold.  bf16: eight roundings of half a step (2^-8) follow one another on the longest way (h, q, tq, o,
# y; dy, do, dq, dh), each of which moves a norm by 2^-8 / sqrt(3) at most, the attention's own tolerance is 2e-2.
TOLERANCE = {"f32": 1e-4, "bf16": 4e-2}


@pytest.mark.parametrize("B,grid,H,d,dtype,norm,extra", [
    (1, (3, 11, 31), 2, 64, "f32", "token", 0), (2, (2, 9, 13), 3, 64, "f32", "head", 5), (1, (3, 9, 17), 2, 128, "bf16", "token", 2),
    (2, (1, 16, 16), 4, 64, "bf16", "head", 0)])
def test_a_layer(B, grid, H, d, dtype, norm, extra):
    import torch
    m = Layer(B, grid, H, d, dtype, norm, extra, block_q=128 if d == 128 else 64)
    got = m.run()
    torch.cuda.synchronize()
    ref = m.reference()
    for name, t in got.items():
        r = float(np.linalg.norm(f64(t) - ref[name]) / np.linalg.norm(ref[name]))
        assert r <= TOLERANCE[dtype], (name, r)


def test_a_captured_layer():
    """The elementwise steps and the attention of a step in one graph, behind products made before: every replay, with the program's own
    work in between, gives the eager bits."""
    import torch
    m = Layer(1, (3, 11, 31), 3, 128, "bf16", "token", extra=4, block_q=128)
    want = {k: t.clone() for k, t in m.run().items()}
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        m.run(side)
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=side):
            got = m.run(side)
    torch.cuda.synchronize()
    scratch = torch.empty(1 << 20, device="cuda")
    for rep in range(4):
        for t in got.values():
            t.fill_(3.0)
        m.ws.random_(0, 255)
        m.aws.random_(0, 255)
        scratch.normal_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for name, t in got.items():
            assert torch.equal(t, want[name]), (rep, name)
