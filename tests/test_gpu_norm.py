"""sla2_norm_forward and sla2_norm_backward through the C ABI against the fp64 statement of the same."""
import numpy as np
import pytest

import layer_oracle as L
from layer_helpers import GUARD, PAD, close, f64, sum_units

pytestmark = pytest.mark.gpu

KINDS, MODS = ["none", "rms", "layer"], ["batch", "token", "shared"]
TYPES = [("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32")]


class Case:
    """Inputs of one call, and the calls.  absent: names among gate, scale, shift, wi, wo that are not given."""

    def __init__(self, B, N, C, x="f32", h="bf16", norm_in="layer", norm_out="none", mods="batch", part="both", rho=1.0, eps=1e-5,
                 absent=(), strided=False, mean=0.5, seed=0):
        import torch
        from paper_2602_12675_amd import api
        self.torch, self.api = torch, api
        self.B, self.N, self.C, self.part, self.rho, self.eps = B, N, C, part, rho, eps
        self.kin, self.kout, self.mods, self.strided = norm_in, norm_out, mods, strided
        ty = {"bf16": torch.bfloat16, "f32": torch.float32}
        self.tx, self.th = ty[x], ty[h]
        g = self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.before, self.after = part != "after", part != "before"
        self.x = self.rows(self.tx, lambda s: 2 * torch.randn(s, generator=g, device="cuda") + mean)
        self.y = self.rows(self.th, lambda s: torch.randn(s, generator=g, device="cuda") - mean) if self.after else None
        m = 0.5 * torch.randn(self.lead() + (6, C), generator=g, device="cuda")
        self.v = {"gate": m[..., 1, :], "scale": m[..., 3, :], "shift": m[..., 4, :]}
        if mods == "shared":
            self.v = {k: t.contiguous() for k, t in self.v.items()}
        self.v["wi"], self.v["wo"] = (1 + 0.3 * torch.randn(C, generator=g, device="cuda") for _ in range(2))
        for name in absent:
            self.v[name] = None
        if not self.before:
            self.v.update(scale=None, shift=None, wi=None)
        if not self.after:
            self.v.update(gate=None, wo=None)
        pad = PAD if strided else 0
        row = (N * (C + pad), C + pad) if not strided else (C + pad, B * (C + pad))          # strided: [N, B, C + pad]
        code = {"bf16": api.SLA2_BF16, "f32": api.SLA2_F32}
        self.p = api.make_norm_params(B, N, C, dtype_x=code[x], dtype_h=code[h], norm_in=KINDS.index(norm_in), norm_out=KINDS.index(norm_out),
                                      eps=eps, residual_scale=rho, mod_layout=MODS.index(mods), x_stride=row, h_stride=row,
                                      mod_stride={"batch": (6 * C, 0), "token": (6 * N * C, 6 * C), "shared": None}[mods])

    def lead(self):
        return {"batch": (self.B,), "token": (self.B, self.N), "shared": ()}[self.mods]

    def rows(self, dtype, make=None):
        """A [B, N, C] view, in a padded [N, B, C + pad] buffer where the case is strided."""
        torch = self.torch
        if self.strided:
            t = torch.full((self.N, self.B, self.C + PAD), GUARD, dtype=dtype, device="cuda")[..., :self.C].transpose(0, 1)
        else:
            t = torch.full((self.B, self.N, self.C), GUARD, dtype=dtype, device="cuda")
        if make is not None:
            t.copy_(make(t.shape))
        return t

    def guard_ok(self, *ts):
        if self.strided:
            for t in ts:
                if t is not None:
                    whole = self.torch.as_strided(t, (self.N, self.B, self.C + PAD), (self.B * (self.C + PAD), self.C + PAD, 1))
                    assert bool((whole[..., self.C:] == GUARD).all())

    def get(self, name):
        t = self.v[name]
        return None if t is None else f64(t)

    def forward(self, x=None, y=None, x_out=None, h=None, **kw):
        x = self.x if x is None else x
        y = self.y if y is None else y
        x_out = (self.rows(self.tx) if x_out is None else x_out) if self.after else None
        h = (self.rows(self.th) if h is None else h) if self.before else None
        v = self.v
        self.api.sla2_norm_forward(self.p, x, h, y=y, x_out=x_out, gate=v["gate"], out_weight=v["wo"], in_weight=v["wi"],
                                   scale=v["scale"], shift=v["shift"], **kw)
        return x_out, h

    def check_forward(self):
        x_out, h = self.forward()
        self.torch.cuda.synchronize()
        x1 = f64(self.x)
        if self.after:
            ref, mag = L.residual(x1, f64(self.y), self.kout, self.rho, self.get("gate"), self.get("wo"), self.mods, self.eps)
            close(x_out, ref, mag, self.tx, what="x_out")
            x1 = f64(x_out)                           # h is taken of what is stored
        if self.before:
            ref, mag = L.before(x1, self.kin, self.get("wi"), self.get("scale"), self.get("shift"), self.mods, self.eps)
            close(h, ref, mag, self.th, what="h")
        self.guard_ok(x_out, h)
        return x_out, h

    def gradients(self, dh, dx_out, x=None, y=None, dx=None, dy=None, ws=None, only=None, **kw):
        """only: the names among dgate, dout_weight, din_weight, dscale, dshift that are wanted (None: all there can be)"""
        torch, v = self.torch, self.v
        x, y = self.x if x is None else x, self.y if y is None else y
        out = {"dx": self.rows(self.tx) if dx is None else dx, "dy": (self.rows(self.th) if dy is None else dy) if self.after else None}
        for name, of in (("dgate", "gate"), ("dscale", "scale"), ("dshift", "shift"), ("dout_weight", "wo"), ("din_weight", "wi")):
            there = self.before and dh is not None if name == "dshift" else v[of] is not None
            if not there or (only is not None and name not in only):
                out[name] = None
            elif of in ("wo", "wi") or self.mods == "shared":
                out[name] = torch.full((self.C,), GUARD, device="cuda")
            else:
                m = torch.full(self.lead() + (6, self.C), GUARD, device="cuda")
                out[name] = m[..., 2, :]
        if ws is None:
            ws = torch.empty(self.api.sla2_norm_workspace_bytes(self.p), dtype=torch.uint8, device="cuda").fill_(255)
        self.api.sla2_norm_backward(self.p, x, dh, dx_out, out["dx"], y=y, gate=v["gate"], out_weight=v["wo"], in_weight=v["wi"],
                                    scale=v["scale"], dy=out["dy"], workspace=ws,
                                    **{k: out[k] for k in ("dgate", "dout_weight", "din_weight", "dscale", "dshift")}, **kw)
        return out

    def incoming(self, residual=True):
        torch, g = self.torch, self.gen
        make = lambda s: torch.randn(s, generator=g, device="cuda")                     # noqa: E731
        return self.rows(self.th, make) if self.before else None, self.rows(self.tx, make) if residual else None

    def check_backward(self, residual=True):
        dh, dx_out = self.incoming(residual)
        out = self.gradients(dh, dx_out)
        self.torch.cuda.synchronize()
        opt = lambda t: None if t is None else f64(t)                                   # noqa: E731
        ref = L.norm_backward(f64(self.x) if self.before else None, opt(self.y), opt(dh), opt(dx_out), self.kin, self.kout, self.rho,
                              self.get("gate"), self.get("wo"), self.get("wi"), self.get("scale"), self.mods, self.eps)
        for name, t in out.items():
            if t is None:
                continue
            summed = name in ("dout_weight", "din_weight") or (name not in ("dx", "dy") and self.mods != "token")
            dt = {"dx": self.tx, "dy": self.th}.get(name, self.torch.float32)
            # a value behind the second norm carries the roundings of the first one's gradient too
            close(t, *ref[name], dt, (sum_units(self.N * (self.B if self.mods == "shared" or "weight" in name else 1)) if summed else 128) +
                  64, name)
        self.guard_ok(out["dx"], out["dy"])
        return dh, dx_out, out


WIDTHS = [8, 16, 24, 64, 72, 128, 320, 512, 520, 1024, 1032, 1536, 2048, 2560, 3584, 4608, 5120, 8192]


@pytest.mark.parametrize("types", TYPES, ids=lambda t: "-".join(t))
@pytest.mark.parametrize("C", WIDTHS)
def test_widths(C, types):
    """Every way that a row is spread over lanes and waves, with all parts there are."""
    k = WIDTHS.index(C)
    for B, N, kin, kout in ((2, 5, "layer", "rms"), (1, 37, "rms", "layer")):
        c = Case(B, N, C, *types, norm_in=kin, norm_out=kout, mods=MODS[(k + B) % 3], rho=0.75, seed=C)
        c.check_forward()
        c.check_backward()


@pytest.mark.parametrize("types", TYPES, ids=lambda t: "-".join(t))
@pytest.mark.parametrize("mods", MODS)
@pytest.mark.parametrize("part", ["before", "after", "both"])
@pytest.mark.parametrize("norm_in,norm_out", [("none", "none"), ("rms", "none"), ("layer", "rms"), ("none", "layer"), ("rms", "rms")])
def test_parts_norms_and_modulations(norm_in, norm_out, part, mods, types):
    c = Case(3, 26, 200, *types, norm_in=norm_in, norm_out=norm_out, mods=mods, part=part, seed=11)
    c.check_forward()
    c.check_backward()
    if part != "after":
        c.check_backward(residual=False)


@pytest.mark.parametrize("absent", [("gate",), ("scale",), ("shift",), ("wi", "wo"), ("gate", "scale", "shift"),
                                    ("gate", "scale", "shift", "wi", "wo")])
@pytest.mark.parametrize("mods", MODS)
def test_absent_vectors(absent, mods):
    c = Case(2, 19, 136, norm_in="layer", norm_out="rms", mods=mods, absent=absent, seed=2)
    c.check_forward()
    c.check_backward()


@pytest.mark.parametrize("B,N,C", [(1, 1, 1536), (7, 1, 64), (1, 1, 8), (600, 1, 128), (600, 3, 40), (1, 1300, 8192), (3, 1111, 1032),
                                   (1, 40000, 8), (2, 700, 5120), (1, 4099, 2048), (65535, 1, 8)])
@pytest.mark.parametrize("mods", ["batch", "shared"])
def test_rows(B, N, C, mods):
    """One row, fewer rows than teams, more batches than workgroups, several rounds of every workgroup with a ragged last one."""
    c = Case(B, N, C, norm_in="rms", norm_out="rms", mods=mods, seed=N)
    c.check_forward()
    c.check_backward()


@pytest.mark.parametrize("N,C", [(127, 8), (128, 8), (129, 8), (3, 72), (33, 136), (16, 264), (17, 264), (5, 1536), (6, 1536), (1, 8192), (2, 8192)])
@pytest.mark.parametrize("mods", MODS)
def test_rows_of_one_workgroup(N, C, mods):
    """As many rows as one workgroup takes side by side, whose sums need no second launch, and one more.  Each gradient alone has the
    bits that it has with all."""
    import torch
    c = Case(1, N, C, norm_in="layer", norm_out="rms", mods=mods)
    dh, dx_out, want = c.check_backward()
    for only in [(n,) for n in ("dgate", "dout_weight", "din_weight", "dscale", "dshift")]:
        got = c.gradients(dh, dx_out, only=only)
        for name in ("dx", "dy") + only:
            assert torch.equal(got[name], want[name]), (only, name)


@pytest.mark.parametrize("types", TYPES, ids=lambda t: "-".join(t))
@pytest.mark.parametrize("C", [64, 1032, 2560])
def test_strides(C, types):
    """[N, B, C] rows with something between them that must be left alone; modulations are slices of [B, 6, C] throughout."""
    for mods in MODS:
        c = Case(3, 21, C, *types, norm_in="layer", norm_out="layer", mods=mods, strided=True, seed=5)
        c.check_forward()
        c.check_backward()


@pytest.mark.parametrize("types", TYPES, ids=lambda t: "-".join(t))
@pytest.mark.parametrize("C", [40, 1536, 5120])
def test_one_call_gives_the_bits_of_two(C, types):
    import torch
    for kin, kout in (("layer", "none"), ("rms", "layer")):
        c = Case(2, 77, C, *types, norm_in=kin, norm_out=kout, rho=1.25)
        x_out, h = c.forward()
        v = c.v
        x2, h2 = torch.empty_like(x_out), torch.empty_like(h)
        c.api.sla2_norm_forward(c.p, c.x, None, y=c.y, x_out=x2, gate=v["gate"], out_weight=v["wo"])
        c.api.sla2_norm_forward(c.p, x2, h2, in_weight=v["wi"], scale=v["scale"], shift=v["shift"])
        assert torch.equal(x_out, x2) and torch.equal(h, h2)


@pytest.mark.parametrize("types", TYPES, ids=lambda t: "-".join(t))
@pytest.mark.parametrize("mods", MODS)
def test_in_place(mods, types):
    import torch
    for C in (72, 2560):
        c = Case(2, 31, C, *types, norm_in="layer", norm_out="rms", mods=mods)
        x_out, h = c.forward()
        x, y = c.x.clone(), c.y.clone()
        c.forward(x=x, y=y, x_out=x, h=y)
        assert torch.equal(x, x_out) and torch.equal(y, h)
        dh, dx_out, want = c.check_backward()
        for over in ("gradients", "values"):
            a, b, gx, gy = c.x.clone(), c.y.clone(), dx_out.clone(), dh.clone()
            got = c.gradients(gy, gx, x=a, y=b, dx=gx if over == "gradients" else a, dy=gy if over == "gradients" else b)
            for name, t in got.items():
                assert torch.equal(t, want[name]), (over, name)


@pytest.mark.parametrize("mods", MODS)
def test_gradients_that_are_not_wanted(mods):
    """Each alone has the bits that it has with all; none at all takes no workspace."""
    import torch
    c = Case(2, 53, 264, norm_in="rms", norm_out="layer", mods=mods)
    dh, dx_out, want = c.check_backward()
    names = ("dgate", "dout_weight", "din_weight", "dscale", "dshift")
    for only in [()] + [(n,) for n in names]:
        got = c.gradients(dh, dx_out, only=only)
        for name in ("dx", "dy") + only:
            assert torch.equal(got[name], want[name]), (only, name)
    dx, dy = c.rows(c.tx), c.rows(c.th)
    v = c.v
    c.api.sla2_norm_backward(c.p, c.x, dh, dx_out, dx, y=c.y, gate=v["gate"], out_weight=v["wo"], in_weight=v["wi"], scale=v["scale"], dy=dy)
    assert torch.equal(dx, want["dx"]) and torch.equal(dy, want["dy"])


def test_constant_and_zero_rows():
    """Rows without spread: the layer norm gives the shift, and its gradient is that of dividing by sqrt(eps)."""
    import torch
    for C in (24, 1536, 4608):
        c = Case(2, 9, C, x="f32", h="f32", norm_in="layer", norm_out="rms", part="before", eps=1e-3)
        c.x[0, 2] = 0
        c.x[1, 4] = 3.0
        _, h = c.check_forward()
        assert torch.equal(h[0, 2], c.v["shift"][0]) and torch.equal(h[1, 4], c.v["shift"][1])
        c.check_backward()


@pytest.mark.parametrize("C", [64, 1032, 5120])
def test_a_mean_that_is_large_beside_the_spread(C):
    """x = 200 +- 2: what single-pass sums of squares in fp32 would lose.  The bound counts 200 r a unit (mag has it)."""
    c = Case(1, 40, C, x="f32", h="f32", norm_in="layer", norm_out="layer", mean=200.0)
    c.check_forward()
    c.check_backward()


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_what_is_not_finite_stays_in_its_row(bad):
    import torch
    for C in (8, 40, 1536):
        c = Case(2, 30, C, norm_in="layer", norm_out="rms")
        x_want, h_want = c.forward()
        dh, dx_out, want = c.check_backward()
        c.y[1, 17, C - 1] = bad
        x_out, h = c.forward()
        keep = torch.ones(2, 30, dtype=torch.bool, device="cuda")
        keep[1, 17] = False
        assert torch.equal(x_out[keep], x_want[keep]) and torch.equal(h[keep], h_want[keep])
        assert not bool(torch.isfinite(h[1, 17]).any())
        got = c.gradients(dh, dx_out)
        assert torch.equal(got["dx"][keep], want["dx"][keep]) and torch.equal(got["dy"][keep], want["dy"][keep])
        assert torch.equal(got["dgate"][0], want["dgate"][0]) and torch.equal(got["dscale"], want["dscale"])


def test_offsets_beyond_32_bits():
    import torch
    from paper_2602_12675_amd import api
    C, N, tok = 136, 4, (1 << 30) + 8
    buf = torch.empty((N - 1) * tok + C, dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(buf, (1, N, C), ((N - 1) * tok + C, tok, 1))
    x.copy_(torch.randn((1, N, C), device="cuda"))
    far = api.make_norm_params(1, N, C, x_stride=(4 * tok, tok), h_stride=(4 * tok, tok))
    near = api.make_norm_params(1, N, C)
    xc, y = x.contiguous(), torch.empty((1, N, C), dtype=torch.bfloat16, device="cuda")
    api.sla2_norm_forward(near, xc, y)
    h = torch.as_strided(torch.empty_like(buf), x.shape, x.stride())
    api.sla2_norm_forward(far, x, h)
    assert torch.equal(h, y)
    dx, want = torch.as_strided(torch.empty_like(buf), x.shape, x.stride()), torch.empty_like(y)
    api.sla2_norm_backward(near, xc, xc, xc, want)
    api.sla2_norm_backward(far, x, x, x, dx)
    assert torch.equal(dx, want)


def test_another_stream_and_a_captured_call():
    """On a side stream, then two calls with workspaces of their own in one graph: every replay gives the eager bits."""
    import torch
    c = Case(2, 300, 1536, norm_in="layer", norm_out="rms", rho=0.5)
    dh, dx_out, want = c.check_backward()
    x_want, h_want = c.forward()
    want = dict(want, x_out=x_want, h=h_want)
    side, got, wss = torch.cuda.Stream(), {}, [torch.empty(c.api.sla2_norm_workspace_bytes(c.p), dtype=torch.uint8, device="cuda")
                                               for _ in range(2)]
    x_out, h = c.rows(c.tx), c.rows(c.th)

    def both(stream):
        c.forward(x_out=x_out, h=h, stream=stream)
        for i, ws in enumerate(wss):
            got[i] = c.gradients(dh, dx_out, ws=ws, stream=stream)

    def check(what):
        torch.cuda.synchronize()
        for i in range(2):
            for name, t in list(got[i].items()) + [("x_out", x_out), ("h", h)]:
                assert torch.equal(t, want[name]), (what, name)
        for i in range(2):
            for t in got[i].values():
                t.fill_(GUARD)
            wss[i].random_(0, 255)
        x_out.fill_(GUARD)
        h.fill_(GUARD)
        torch.cuda.synchronize()

    with torch.cuda.stream(side):
        side.wait_stream(torch.cuda.default_stream())
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


def test_weights_gradients_over_many_rows_against_differences():
    """d w_in, d scale and d gate by differences of a loss in fp64 made of the library's own forward results."""
    import torch
    c = Case(1, 64, 64, x="f32", h="f32", norm_in="rms", norm_out="layer")
    dh, dx_out = c.incoming()
    x_out, h = c.forward()
    got = c.gradients(dh, dx_out, x=x_out)

    def loss():
        a, b = c.forward()
        return float((a.double() * dx_out.double()).sum() + (b.double() * dh.double()).sum())

    step = 2.0 ** -6                                  # results are rounded to 2^-24 of themselves: sums of 8192 of them to about 1e-4
    for name, of in (("din_weight", "wi"), ("dscale", "scale"), ("dgate", "gate"), ("dout_weight", "wo"), ("dshift", "shift")):
        t = c.v[of]
        for at in (0, 31, 63):
            i = (at,) if t.dim() == 1 else (0, at)
            old = float(t[i])
            t[i] = old + step
            up = loss()
            t[i] = old - step
            down = loss()
            t[i] = old
            want = float(got[name][i])
            assert abs((up - down) / (2 * step) - want) <= 2e-2 * max(1.0, abs(want)), (name, at)
