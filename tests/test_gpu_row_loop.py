"""Rows that a team takes one after the other: sizes at which every workgroup of sla2_rope_* and sla2_norm_* goes round its loop several times,
the last time with rows left for some of its teams only (tests/test_row_plan.py checks that they do, by the plans themselves); and sums over
rows whose terms are whole numbers, so that they are exact whatever their order and a row that is left out or taken twice shows.

The bounds of values are ROW_UNITS of layer_helpers.  They cover rows of three chunks a thread: a sum has 24 terms in turn in a lane, 6 steps over
the lanes and 4 over the waves, its mean 2 roundings more, 36 in all, of which a root passes on half, with 3 of its own; a result has fewer
than 24 of its own."""
import pytest

import test_gpu_norm as NT
import test_gpu_rope as RT

pytestmark = pytest.mark.gpu

# B, H, N, d, positions: None: given, else the grid.  A step of the grid goes on in x, in y and in t, tokens past it come on a later step.
ROPE = [
    (257, 1, 150, 64, (5, 4, 7)),            # 64 teams of 8 lanes a workgroup
    (130, 2, 107, 64, None),                 # 16 lanes
    (257, 3, 35, 64, (2, 3, 5)),             # 24 of 32 lanes
    (257, 1, 70, 128, (3, 4, 5)),
    (257, 5, 19, 64, (1, 3, 6)),             # a wave
    (1, 12, 4200, 128, (9, 15, 31)),         # three chunks a thread, forward; three waves, backward
    (3, 20, 1400, 64, (3, 14, 33)),          # of three waves the last half empty, backward
    (2, 40, 1100, 128, None),                # 640 chunks: four waves of three, forward; ten waves, backward
    (520, 64, 3, 128, (1, 1, 2)),            # 16 waves, backward: one row a workgroup
]
WAYS = [("token", False, "bf16"), ("token", True, "f32"), ("head", True, "bf16"), ("head", False, "f32"), ("none", False, "bf16"), ("none", True, "f32")]


@pytest.mark.parametrize("size", ROPE, ids=lambda s: "x".join(map(str, s[:4])))
@pytest.mark.parametrize("way", WAYS, ids=lambda w: "-".join(map(str, w)))
def test_rope(size, way):
    B, H, N, d, grid = size
    norm, halves, dtype = way
    c = RT.Case(B, H, N, d, dtype=dtype, halves=halves, norm=norm, grid=grid, origin=(3, -2, 40) if grid else (0, 0, 0), seed=N,
                layout="tokens" if halves else "packed", out_layout="tokens")
    c.check_forward()
    c.check_backward()


# B, N, C
NORM = [
    (257, 150, 8),                           # 64 teams of 8 lanes, one of which has channels
    (257, 70, 72),                           # 9 of 16 lanes
    (257, 35, 200),                          # 25 of 32
    (257, 19, 520),                          # a wave and a chunk: two a thread, forward; two waves, backward
    (1, 4200, 1536),                         # three a thread, forward; three waves, backward
    (257, 9, 2560),                          # two waves of three, forward; five waves, backward
    (257, 3, 8192),                          # six waves of three, forward; 16 waves, backward
]
FORMS = [("f32", "bf16", "layer", "none", "batch", "both"), ("bf16", "bf16", "layer", "rms", "token", "both"), ("f32", "f32", "rms", "layer", "shared", "both"),
         ("f32", "bf16", "layer", "none", "token", "before"), ("bf16", "bf16", "rms", "none", "batch", "before"),
         ("f32", "bf16", "none", "layer", "token", "after"), ("f32", "f32", "none", "rms", "batch", "after")]


@pytest.mark.parametrize("size", NORM, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("form", FORMS, ids="-".join)
def test_norm(size, form):
    x, h, kin, kout, mods, part = form
    c = NT.Case(*size, x=x, h=h, norm_in=kin, norm_out=kout, mods=mods, part=part, rho=0.75, seed=size[1])
    c.check_forward()
    c.check_backward()


# ---- sums that are exact ----
SUMS = [(1, 40000, 8), (65535, 1, 8), (600, 40, 136), (3, 4111, 1032), (1, 9001, 1536), (257, 9, 2560), (5, 700, 5120), (1, 1300, 8192)]


@pytest.mark.parametrize("part", ["before", "after", "both"])
@pytest.mark.parametrize("mods", NT.MODS)
@pytest.mark.parametrize("B,N,C", SUMS)
def test_sums_of_whole_numbers(B, N, C, mods, part):
    """Without norms, every value a small whole number: |u| <= 2 + 2 x 2 x 3, |u y g| <= 14 x 2 x 2 = 56, 56 x 65,535 < 2^24, so each sum is exact in
    fp32 in any order, and the fp64 sum has the same value."""
    import torch
    c = NT.Case(B, N, C, x="f32", h="bf16", norm_in="none", norm_out="none", mods=mods, part=part)
    g = torch.Generator(device="cuda").manual_seed(N)
    whole = lambda like, lo, hi: like.copy_(torch.randint(lo, hi + 1, like.shape, generator=g, device="cuda"))        # noqa: E731
    for name, lo, hi in (("gate", 1, 2), ("scale", 0, 2), ("shift", -2, 2), ("wi", 1, 2), ("wo", 1, 1)):
        if c.v[name] is not None:
            whole(c.v[name], lo, hi)
    whole(c.x, 1, 2)
    if c.after:
        whole(c.y, 1, 2)
    dh, dx_out = c.incoming()
    for t in (dh, dx_out):
        if t is not None:
            whole(t, 1, 2)                   # no term is 0
    out = c.gradients(dh, dx_out)
    torch.cuda.synchronize()
    dbl = lambda t: None if t is None else t.double()                                                              # noqa: E731
    wide = lambda m: m[:, None] if mods == "batch" else m                                                          # noqa: E731
    to_mod = lambda t: t if mods == "token" else t.sum(1) if mods == "batch" else t.sum((0, 1))                     # noqa: E731
    want, u = {}, dbl(dx_out)
    if c.before:
        s, w, d, x = wide(dbl(c.v["scale"])), dbl(c.v["wi"]), dbl(dh), dbl(c.x)
        want["dshift"], want["dscale"], want["din_weight"] = to_mod(d), to_mod(d * x * w), (d * x * (1 + s)).sum((0, 1))
        u = u + d * w * (1 + s)
    if c.after:
        gate, w, y = wide(dbl(c.v["gate"])), dbl(c.v["wo"]), dbl(c.y)
        want["dgate"], want["dout_weight"], want["dy"] = to_mod(u * y * w), (u * y * gate).sum((0, 1)), u * gate * w
    want["dx"] = u
    for name, t in want.items():
        assert float(t.abs().max()) <= 2 ** 24
        assert torch.equal(out[name].double(), t), name


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("norm", ["head", "token"])
@pytest.mark.parametrize("B,H,N,d", [s[:4] for s in ROPE] + [(1, 1, 40000, 64), (65535, 1, 1, 64), (1, 12, 32760, 128), (300, 3, 40, 128), (1, 1, 70, 128)])
def test_sums_of_whole_numbers_of_the_norm_of_q_and_k(B, H, N, d, norm, dtype):
    """x = +-1 and the smallest eps: the root is 1; positions of 0: nothing turns.  Then dw is the sum of dy x, whole numbers that are not 0, at
    most 2 x 32,760 x 12 in all: exact in fp32 in any order."""
    import torch
    c = RT.Case(B, H, N, d, dtype=dtype, norm=norm, layout="tokens", positions=torch.zeros((1, N, 3), device="cuda"), per_batch=0, eps=2.0 ** -126)
    sign = lambda t: t.copy_(torch.randint(0, 2, t.shape, generator=c.gen, device="cuda") * 2 - 1)                  # noqa: E731
    sign(c.q)
    sign(c.k)
    gq, gk, dq, dk = (torch.empty_like(c.q) for _ in range(4))
    for g in (gq, gk):
        sign(g).mul_(torch.randint(1, 3, g.shape, generator=c.gen, device="cuda"))
    dw = [torch.full_like(c.w[0], RT.GUARD) for _ in range(2)]
    ws = torch.empty(c.api.sla2_rope_workspace_bytes(c.p), dtype=torch.uint8, device="cuda").fill_(255)
    p = c.api.make_rope_params(B, H, N, d, c.axes, dtype=c.p.dtype, norm=c.p.norm, eps=2.0 ** -126, in_stride=c.ist, out_stride=c.ist)
    c.api.sla2_rope_backward(p, c.q, c.k, c.freq, gq, gk, dq, dk, q_weight=c.w[0], k_weight=c.w[1], dq_weight=dw[0], dk_weight=dw[1],
                             positions=c.pos, workspace=ws)
    for x, g, got in ((c.q, gq, dw[0]), (c.k, gk, dw[1])):
        want = (x.double() * g.double()).sum((0, 1, 2) if norm == "head" else (0, 2))
        assert torch.equal(got.double(), want)
