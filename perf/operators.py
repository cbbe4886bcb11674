"""Performance cases of the steps around the attention of a diffusion transformer's layer: rotary positions of q and k
with several axes, and the norms before and after a block with its modulation, gate and residual.

A case is a dict of plain values.  kind "rope" (forward) and "rope_bwd":
  B, H, N, d     q and k are [B, H, N, d] views
  dtype          "bf16" | "f32"        element type of q, k and the results
  layout         "packed"  q, k are slices of one [B, N, 3, H, d] projection, results are [B, N, H, d]
                 "tokens"  all are [B, N, H, d]           "heads"  all are [B, H, N, d]
  grid           "T,Y,X": token n is at (n / (Y X), n / X % Y, n % X), tokens past the grid are not rotated;
                 "": int32 positions [B, N, 3] are given
  axes           "a,b,c": rotated pairs of the time, height and width axis
  pairing        "interleaved" pair j is channels (2 j, 2 j + 1) | "halves" (j, j + d / 2)
  norm           "none" | "head" RMS norm over the d channels of a head | "token" over the H d channels of a token
kind "norm" (forward) and "norm_bwd":
  B, N, C        x, y, h are [B, N, C]
  x, h           element type of the residual stream x, and of the block's output y and input h
  part           "both"    x' = rho x + gate (.) norm_out(y), h = norm_in(x') (.) (1 + scale) + shift
                 "before"  h alone, x' = x         "after"  x' alone
  norm_in, norm_out    "none" | "rms" | "layer"
  mods           gate, scale and shift are slices of "batch" [B, 3, C], "token" [B, N, 3, C], "shared" [3, C]
  weights        whether the norms have a weight [C]
  rho            scale of the residual
"""
import math

import torch

own = False

EPS = 1e-6
THETA = 10000.0


def _rope(name, kind, B, H, N, d, dtype, layout, grid, axes, pairing, norm):
    return {"name": name, "kind": kind, "B": B, "H": H, "N": N, "d": d, "dtype": dtype, "layout": layout, "grid": grid, "axes": axes,
            "pairing": pairing, "norm": norm}


def _norm(name, kind, B, N, C, x, h, part, norm_in, norm_out, mods, weights, rho=1.0):
    return {"name": name, "kind": kind, "B": B, "N": N, "C": C, "x": x, "h": h, "part": part, "norm_in": norm_in, "norm_out": norm_out,
            "mods": mods, "weights": weights, "rho": rho}


def listed():
    return [
        # one token of a stream, behind the projection of a 12-head model: nothing but latency
        _rope("rope-one-token", "rope", 1, 12, 1, 128, "bf16", "packed", "", "22,21,21", "interleaved", "token"),
        # fp32 reference runs of an image model, 64 x 64 latents, a guidance pair
        _rope("rope-image-4k-f32", "rope", 2, 16, 4096, 64, "f32", "heads", "1,64,64", "0,16,16", "halves", "head"),
        # one layer of video generation on the 21 x 30 x 52 grid, out of the packed projection
        _rope("rope-wan1.3b", "rope", 1, 12, 32760, 128, "bf16", "packed", "21,30,52", "22,21,21", "interleaved", "token"),
        # 720p video on the 21 x 45 x 80 grid and one token past it, q and k from projections of their own
        _rope("rope-wan14b-ragged", "rope", 1, 40, 75601, 128, "bf16", "tokens", "21,45,80", "22,21,21", "interleaved", "token"),
        # training of the smaller video model
        _rope("rope-bwd-wan1.3b", "rope_bwd", 1, 12, 32760, 128, "bf16", "tokens", "21,30,52", "22,21,21", "interleaved", "token"),
        # training with text and image tokens in one sequence, positions given, odd length
        _rope("rope-bwd-joint-image", "rope_bwd", 2, 20, 4429, 64, "bf16", "packed", "", "8,12,12", "halves", "head"),
        # one token a sequence, a guidance pair: latency of the step between two blocks
        _norm("norm-one-token", "norm", 2, 1, 1536, "f32", "bf16", "both", "layer", "rms", "batch", True),
        # before the first block of the smaller video model, residual stream in fp32
        _norm("norm-before-wan1.3b", "norm", 1, 32760, 1536, "f32", "bf16", "before", "layer", "none", "batch", False),
        # between two blocks of the larger one
        _norm("norm-both-wan14b", "norm", 1, 75600, 5120, "f32", "bf16", "both", "layer", "none", "batch", False),
        # a time step of its own for every token (frames that are given beside frames that are made), norms on both sides
        _norm("norm-per-token", "norm", 2, 12481, 2048, "bf16", "bf16", "both", "rms", "rms", "token", True),
        # training of the smaller video model, a frame missing
        _norm("norm-bwd-wan1.3b", "norm_bwd", 1, 31201, 1536, "f32", "bf16", "both", "layer", "none", "batch", False),
        # fp32 reference training of an image model with learned norms and layer scale
        _norm("norm-bwd-image-f32", "norm_bwd", 2, 4096, 1152, "f32", "f32", "both", "rms", "rms", "shared", True, 0.5),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Work up to that of the largest listed case, which is 75,600 rows of 5,120 channels, with three sizes of element."""
    if rng.random() < 0.5:
        kind, d, H = rng.choice(["rope", "rope_bwd"]), rng.choice([64, 128]), rng.randint(1, 40)
        B = rng.choice([1, 1, 2, 4])
        N = _log_int(rng, 1, max(1, min(75601, int(1.5e8 / (B * H * d)))))
        pairs = d // 2
        a = rng.choice([0, pairs // 4, pairs - 2 * (pairs // 3)])
        b = (pairs - a) // 2 - rng.choice([0, 0, 3])
        Y, X = rng.randint(1, 48), rng.randint(1, 80)
        grid = rng.choice(["", "%d,%d,%d" % (max(1, N // (Y * X)), Y, X)])
        c = _rope("", kind, B, H, N, d, rng.choice(["bf16", "bf16", "f32"]), rng.choice(["packed", "tokens", "heads"]), grid,
                  "%d,%d,%d" % (a, b, b), rng.choice(["interleaved", "halves"]), rng.choice(["none", "head", "token"]))
    else:
        kind, C = rng.choice(["norm", "norm_bwd"]), 8 * _log_int(rng, 8, 1024)
        B = rng.choice([1, 1, 2, 4])
        x, h = rng.choice([("f32", "bf16"), ("bf16", "bf16"), ("f32", "f32")])
        mods = rng.choice(["batch", "batch", "token", "shared"])
        N = _log_int(rng, 1, max(1, min(75600, int((4e7 if mods == "token" else 1e8) / (B * C)))))
        c = _norm("", kind, B, N, C, x, h, rng.choice(["both", "both", "before", "after"]), rng.choice(["rms", "layer"]),
                  rng.choice(["none", "rms", "layer"]), mods, rng.random() < 0.5, rng.choice([1.0, 0.75]))
    del c["name"]
    return c


def _type(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _three(text):
    return [int(t) for t in text.split(",")] if text else [0, 0, 0]


def _normal(gen, shape, dtype, by=1.0, mean=0.0):
    """Normal values whose spread differs from channel to channel, as activations of a trained model have it."""
    x = torch.randn(shape, generator=gen, device="cuda")
    x *= by * torch.exp(0.5 * torch.randn(shape[-1], generator=gen, device="cuda"))
    return (x + mean).to(dtype) if mean else x.to(dtype)


def _tensors(gen, case):
    """q and k (or gradients of their results) as [B, H, N, d] views, with buffers of the same layout."""
    B, H, N, d, dt = case["B"], case["H"], case["N"], case["d"], _type(case["dtype"])
    if case["layout"] == "packed":
        t = _normal(gen, (B, N, 3, H, d), dt)
        return t[:, :, 0].transpose(1, 2), t[:, :, 1].transpose(1, 2)
    if case["layout"] == "tokens":
        return tuple(_normal(gen, (B, N, H, d), dt).transpose(1, 2) for _ in range(2))
    return tuple(_normal(gen, (B, H, N, d), dt) for _ in range(2))


def _results(case):
    """Buffers of the results: of the layout of the inputs, or [B, N, H, d] where those are packed."""
    B, H, N, d, dt = case["B"], case["H"], case["N"], case["d"], _type(case["dtype"])
    if case["layout"] == "heads":
        return tuple(torch.empty((B, H, N, d), dtype=dt, device="cuda") for _ in range(2))
    return tuple(torch.empty((B, N, H, d), dtype=dt, device="cuda").transpose(1, 2) for _ in range(2))


def _prepare_rope(case, gen):
    B, H, N, d, dt = case["B"], case["H"], case["N"], case["d"], _type(case["dtype"])
    s = {"case": case}
    s["q"], s["k"] = _tensors(gen, case)
    shape = {"none": None, "head": (d,), "token": (H, d)}[case["norm"]]
    if shape:
        s["qw"], s["kw"] = (1.0 + 0.2 * torch.randn(shape, generator=gen, device="cuda") for _ in range(2))
    a = _three(case["axes"])
    s["freq"] = torch.cat([THETA ** (-torch.arange(n, dtype=torch.float64) / max(n, 1)) for n in a] +
                          [torch.zeros(d // 2 - sum(a), dtype=torch.float64)]).cuda()
    if not case["grid"]:
        # frame, row and column of tokens of several pictures in a row, text tokens (all three alike) among them
        base = torch.randint(0, 2000, (B, N, 1), generator=gen, device="cuda")
        off = torch.randint(0, 64, (B, N, 3), generator=gen, device="cuda")
        s["pos"] = torch.where(torch.rand((B, N, 1), generator=gen, device="cuda") < 0.1, base, off).int()
    if case["kind"] == "rope":
        s["out"] = _results(case)
    else:
        s["dout"] = tuple(_normal(gen, (B, H, N, d), dt, 0.1) if case["layout"] == "heads" else
                          _normal(gen, (B, N, H, d), dt, 0.1).transpose(1, 2) for _ in range(2))
        if case["layout"] == "packed":                 # gradients go into one packed buffer, as the projection's backward reads it
            t = torch.empty((B, N, 3, H, d), dtype=dt, device="cuda")
            s["out"] = t[:, :, 0].transpose(1, 2), t[:, :, 1].transpose(1, 2)
        else:
            s["out"] = _results(case)
        if shape:
            s["dw"] = tuple(torch.empty(shape, device="cuda") for _ in range(2))
    if own:
        from paper_2602_12675_amd import api
        tok, hd = (N * H * d, d, H * d), (H * N * d, N * d, d)
        first = {"packed": (N * 3 * H * d, d, 3 * H * d), "tokens": tok, "heads": hd}[case["layout"]]
        s["params"] = api.make_rope_params(
            B, H, N, d, tuple(a), grid=tuple(_three(case["grid"])), dtype=api.SLA2_BF16 if case["dtype"] == "bf16" else api.SLA2_F32,
            pairing={"interleaved": api.SLA2_ROPE_INTERLEAVED, "halves": api.SLA2_ROPE_HALVES}[case["pairing"]],
            norm={"none": api.SLA2_ROPE_NORM_NONE, "head": api.SLA2_ROPE_NORM_HEAD, "token": api.SLA2_ROPE_NORM_TOKEN}[case["norm"]],
            eps=EPS, positions_per_batch=1, in_stride=first, out_stride=hd if case["layout"] == "heads" else tok)
        if "dw" in s:
            s["workspace"] = torch.empty(api.sla2_rope_workspace_bytes(s["params"]), dtype=torch.uint8, device="cuda")
    return s


def _prepare_norm(case, gen):
    B, N, C, tx, th = case["B"], case["N"], case["C"], _type(case["x"]), _type(case["h"])
    s, part, bwd = {"case": case}, case["part"], case["kind"] == "norm_bwd"
    lead = {"batch": (B,), "token": (B, N), "shared": ()}[case["mods"]]
    m = 0.3 * torch.randn(lead + (3, C), generator=gen, device="cuda")
    s["gate"], s["scale"], s["shift"] = m[..., 0, :], m[..., 1, :], m[..., 2, :]
    if part != "after" or not bwd:
        s["x"] = _normal(gen, (B, N, C), tx, 2.0, 0.25)           # backward: what norm_in was taken of
    if part != "before":
        s["y"] = _normal(gen, (B, N, C), th)
    if case["weights"]:
        s["wi"], s["wo"] = (1.0 + 0.2 * torch.randn(C, generator=gen, device="cuda") for _ in range(2))
    if bwd:
        if part != "after":
            s["dh"] = _normal(gen, (B, N, C), th, 0.1)
        s["dx_out"] = _normal(gen, (B, N, C), tx, 0.1)
        s["dx"] = torch.empty((B, N, C), dtype=tx, device="cuda")
        d = torch.empty(lead + (3, C), device="cuda")
        s["dgate"], s["dscale"], s["dshift"] = d[..., 0, :], d[..., 1, :], d[..., 2, :]
        s["dwi"], s["dwo"] = (torch.empty(C, device="cuda") for _ in range(2))
        if part != "before":
            s["dy"] = torch.empty((B, N, C), dtype=th, device="cuda")
    else:
        if part != "before":
            s["x_out"] = torch.empty((B, N, C), dtype=tx, device="cuda")
        if part != "after":
            s["h"] = torch.empty((B, N, C), dtype=th, device="cuda")
    if own:
        from paper_2602_12675_amd import api
        kinds = {"none": api.SLA2_NORM_NONE, "rms": api.SLA2_NORM_RMS, "layer": api.SLA2_NORM_LAYER}
        types = {"bf16": api.SLA2_BF16, "f32": api.SLA2_F32}
        s["params"] = api.make_norm_params(
            B, N, C, dtype_x=types[case["x"]], dtype_h=types[case["h"]], norm_in=kinds[case["norm_in"]], norm_out=kinds[case["norm_out"]],
            eps=EPS, residual_scale=case["rho"],
            mod_layout={"batch": api.SLA2_MOD_BATCH, "token": api.SLA2_MOD_TOKEN, "shared": api.SLA2_MOD_SHARED}[case["mods"]],
            mod_stride={"batch": (3 * C, 0), "token": (N * 3 * C, 3 * C), "shared": (0, 0)}[case["mods"]])
        if bwd:
            s["workspace"] = torch.empty(api.sla2_norm_workspace_bytes(s["params"]), dtype=torch.uint8, device="cuda")
    return s


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (_prepare_rope if case["kind"].startswith("rope") else _prepare_norm)(case, gen)


# ---- the plain forms: elementary operations in 32 bits ----

def _angles(s):
    """[B or 1, N, d / 2]: the angle of every pair, in 64 bits."""
    case = s["case"]
    a, (T, Y, X) = _three(case["axes"]), _three(case["grid"])
    rest = case["d"] // 2 - sum(a)
    axis = torch.repeat_interleave(torch.arange(3), torch.tensor([a[0], a[1], a[2] + rest])).cuda()     # freq is 0 from the axes' end on
    if case["grid"]:
        n = torch.arange(case["N"], device="cuda")
        pos = torch.stack([n // (Y * X), n // X % Y, n % X], -1)
        pos = torch.where((n < T * Y * X)[:, None], pos, 0)[None]
    else:
        pos = s["pos"]
    return pos.double()[..., axis] * s["freq"]


def _pairs(case, x):
    """The two channels of every pair, [..., d / 2] each."""
    return (x[..., 0::2], x[..., 1::2]) if case["pairing"] == "interleaved" else x.chunk(2, -1)


def _unpair(case, a, b):
    return torch.stack([a, b], -1).flatten(-2) if case["pairing"] == "interleaved" else torch.cat([a, b], -1)


def _turn(case, x, c, s):
    a, b = _pairs(case, x)
    return _unpair(case, a * c - b * s, a * s + b * c)


def _root(case, x):
    """What the RMS norm multiplies with, [B, H or 1, N, 1]."""
    dims = (3,) if case["norm"] == "head" else (1, 3)
    return torch.rsqrt((x * x).mean(dims, keepdim=True) + EPS)


def _weight(case, w):
    return w if case["norm"] == "head" else w[:, None, :]


def _plain_rope(s):
    case = s["case"]
    angle = _angles(s)
    c, si = angle.cos().float()[:, None], angle.sin().float()[:, None]

    def one(x, w):
        x = x.float()
        if case["norm"] != "none":
            x = x * _root(case, x) * _weight(case, w)
        return _turn(case, x, c, si).to(_type(case["dtype"]))

    return {"q": one(s["q"], s.get("qw")), "k": one(s["k"], s.get("kw"))}


def _plain_rope_bwd(s):
    case = s["case"]
    angle = _angles(s)
    c, si = angle.cos().float()[:, None], angle.sin().float()[:, None]

    def one(x, w, g):
        g = _turn(case, g.float(), c, -si)
        if case["norm"] == "none":
            return g.to(_type(case["dtype"])), None
        x = x.float()
        r = _root(case, x)
        n = x * r
        dw = (g * n).sum((0, 1, 2) if case["norm"] == "head" else (0, 2))
        g = g * _weight(case, w)
        m = (g * n).mean((3,) if case["norm"] == "head" else (1, 3), keepdim=True)
        return (r * (g - n * m)).to(_type(case["dtype"])), dw

    dq, dqw = one(s["q"], s.get("qw"), s["dout"][0])
    dk, dkw = one(s["k"], s.get("kw"), s["dout"][1])
    out = {"dq": dq, "dk": dk}
    return out if dqw is None else dict(out, dqw=dqw, dkw=dkw)


def _rows(case, m):
    """A modulation as it meets [B, N, C]."""
    return m[:, None] if case["mods"] == "batch" else m


def _standard(kind, x):
    """(normalised x, what it was multiplied with)"""
    if kind == "none":
        return x, None
    if kind == "layer":
        x = x - x.mean(-1, keepdim=True)
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    return x * r, r


def _back(kind, n, r, g):
    """The gradient behind a norm from that in front of it."""
    if kind == "none":
        return g
    m = n * (g * n).mean(-1, keepdim=True)
    return r * (g - m - g.mean(-1, keepdim=True)) if kind == "layer" else r * (g - m)


def _plain_norm(s):
    case, out = s["case"], {}
    x = s["x"].float()
    if case["part"] != "before":
        m, r = _standard(case["norm_out"], s["y"].float())
        if "wo" in s and r is not None:
            m = m * s["wo"]
        out["x_out"] = (case["rho"] * x + _rows(case, s["gate"]) * m).to(s["x"].dtype)
        x = out["x_out"].float()
    if case["part"] != "after":
        n, r = _standard(case["norm_in"], x)
        if "wi" in s:
            n = n * s["wi"]
        out["h"] = (n * (1 + _rows(case, s["scale"])) + _rows(case, s["shift"])).to(_type(case["h"]))
    return out


def _to_mod(case, g):
    """The gradient of a modulation from its terms, [B, N, C]."""
    return g if case["mods"] == "token" else g.sum(1) if case["mods"] == "batch" else g.sum((0, 1))


def _plain_norm_bwd(s):
    case, out = s["case"], {}
    u = s["dx_out"].float()
    if case["part"] != "after":
        n, r = _standard(case["norm_in"], s["x"].float())
        g = s["dh"].float()
        w = s.get("wi")
        out["dshift"] = _to_mod(case, g)
        out["dscale"] = _to_mod(case, g * n if w is None else g * n * w)
        g = g * (1 + _rows(case, s["scale"]))
        if w is not None:
            out["dwi"] = (g * n).sum((0, 1))
            g = g * w
        u = u + _back(case["norm_in"], n, r, g)
    if case["part"] != "before":
        n, r = _standard(case["norm_out"], s["y"].float())
        w = s.get("wo") if r is not None else None
        out["dgate"] = _to_mod(case, u * n if w is None else u * n * w)
        g = u * _rows(case, s["gate"])
        if w is not None:
            out["dwo"] = (g * n).sum((0, 1))
            g = g * w
        out["dy"] = _back(case["norm_out"], n, r, g).to(_type(case["h"]))
        u = case["rho"] * u
    out["dx"] = u.to(_type(case["x"]))
    return out


# ---- the framework's calls ----

def _own_rope(s):
    from paper_2602_12675_amd import api
    q, k = s["out"]
    api.sla2_rope_forward(s["params"], s["q"], s["k"], s["freq"], q, k, q_weight=s.get("qw"), k_weight=s.get("kw"),
                          positions=s.get("pos"))
    return {"q": q, "k": k}


def _own_rope_bwd(s):
    from paper_2602_12675_amd import api
    dq, dk = s["out"]
    dqw, dkw = s.get("dw", (None, None))
    api.sla2_rope_backward(s["params"], s["q"], s["k"], s["freq"], s["dout"][0], s["dout"][1], dq, dk, q_weight=s.get("qw"),
                           k_weight=s.get("kw"), dq_weight=dqw, dk_weight=dkw, positions=s.get("pos"), workspace=s.get("workspace"))
    out = {"dq": dq, "dk": dk}
    return out if dqw is None else dict(out, dqw=dqw, dkw=dkw)


def _own_norm(s):
    from paper_2602_12675_amd import api
    case, before, after = s["case"], s["case"]["part"] != "after", s["case"]["part"] != "before"
    api.sla2_norm_forward(s["params"], s["x"], s.get("h"), y=s.get("y"), x_out=s.get("x_out"), gate=s["gate"] if after else None,
                          out_weight=s.get("wo") if after and case["norm_out"] != "none" else None,
                          in_weight=s.get("wi") if before else None, scale=s["scale"] if before else None,
                          shift=s["shift"] if before else None)
    return {name: s[name] for name in ("x_out", "h") if name in s}


def _own_norm_bwd(s):
    from paper_2602_12675_amd import api
    case, before, after = s["case"], s["case"]["part"] != "after", s["case"]["part"] != "before"
    wi = s.get("wi") if before else None
    wo = s.get("wo") if after and case["norm_out"] != "none" else None
    given = {"dx": s["dx"]}
    if before:
        given.update(dscale=s["dscale"], dshift=s["dshift"])
    if after:
        given.update(dy=s["dy"], dgate=s["dgate"])
    if wi is not None:
        given["dwi"] = s["dwi"]
    if wo is not None:
        given["dwo"] = s["dwo"]
    api.sla2_norm_backward(s["params"], s.get("x"), s.get("dh"), s["dx_out"], s["dx"], y=s.get("y"), gate=s["gate"] if after else None,
                           out_weight=wo, in_weight=wi, scale=s["scale"] if before else None, dy=given.get("dy"),
                           dgate=given.get("dgate"), dout_weight=given.get("dwo"), din_weight=given.get("dwi"),
                           dscale=given.get("dscale"), dshift=given.get("dshift"), workspace=s["workspace"])
    return given


def run(s):
    kind = s["case"]["kind"]
    if own:
        return {"rope": _own_rope, "rope_bwd": _own_rope_bwd, "norm": _own_norm, "norm_bwd": _own_norm_bwd}[kind](s)
    return {"rope": _plain_rope, "rope_bwd": _plain_rope_bwd, "norm": _plain_norm, "norm_bwd": _plain_norm_bwd}[kind](s)


def work(case):
    size = {"bf16": 2, "f32": 4}
    if case["kind"].startswith("rope"):
        n = 2 * case["B"] * case["H"] * case["N"] * case["d"]                    # elements of q and k
        w = {"none": 0, "head": 2 * case["d"], "token": 2 * case["H"] * case["d"]}[case["norm"]] * 4
        pos = 0 if case["grid"] else case["B"] * case["N"] * 12
        normed = case["norm"] != "none"
        if case["kind"] == "rope":
            return {"bytes": 2 * n * size[case["dtype"]] + w + pos, "flops": n * (3 + 4 * normed)}
        return {"bytes": (2 + normed) * n * size[case["dtype"]] + 2 * w + pos, "flops": n * (3 + 10 * normed)}
    n, ex, eh, part = case["B"] * case["N"] * case["C"], size[case["x"]], size[case["h"]], case["part"]
    vectors = (0 if part == "before" else 1) + (0 if part == "after" else 2)     # gate; scale and shift
    mods = vectors * 4 * {"batch": case["B"] * case["C"], "token": n, "shared": case["C"]}[case["mods"]]
    weights = 4 * case["C"] * ((part != "after") + (part != "before" and case["norm_out"] != "none")) if case["weights"] else 0
    if case["kind"] == "norm":
        return {"bytes": n * {"both": 2 * ex + 2 * eh, "before": ex + eh, "after": 2 * ex + eh}[part] + mods + weights,
                "flops": n * {"both": 16, "before": 9, "after": 7}[part]}
    reads = mods - (4 * {"batch": case["B"] * case["C"], "token": n, "shared": case["C"]}[case["mods"]] if part != "after" else 0)   # not the shift
    return {"bytes": n * {"both": 3 * ex + 3 * eh, "before": 3 * ex + eh, "after": 2 * ex + 2 * eh}[part] + reads + mods + 2 * weights,
            "flops": n * {"both": 32, "before": 18, "after": 14}[part]}


# ---- the definitions in 64 bits: rotations as products of complex numbers, gradients by differentiation ----

def _exact_rope(s):
    case = s["case"]
    B, H, N, d = case["B"], case["H"], case["N"], case["d"]
    a, (T, Y, X) = _three(case["axes"]), _three(case["grid"])
    if case["grid"]:
        t, y, x = torch.meshgrid(torch.arange(T), torch.arange(Y), torch.arange(X), indexing="ij")
        pos = torch.zeros((max(N, T * Y * X), 3), dtype=torch.float64)
        pos[:T * Y * X] = torch.stack([t.flatten(), y.flatten(), x.flatten()], 1).double()
        pos = pos[None, :N].cuda()
    else:
        pos = s["pos"].double()
    first, turns = 0, []
    for i in range(3):
        turns.append(pos[:, :, i, None] * s["freq"][first:first + a[i]])
        first += a[i]
    turns.append(torch.zeros(turns[0].shape[:2] + (d // 2 - first,), dtype=torch.float64, device="cuda"))
    unit = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), torch.cat(turns, -1))[:, None]

    def one(x, w):
        if case["norm"] == "head":
            x = x / (x.pow(2).sum(-1, keepdim=True) / d + EPS).sqrt() * w
        elif case["norm"] == "token":
            x = x / (x.pow(2).sum((1, 3), keepdim=True) / (H * d) + EPS).sqrt() * w.view(1, H, 1, d)
        inter = case["pairing"] == "interleaved"
        z = x.reshape(B, H, N, d // 2, 2) if inter else x.reshape(B, H, N, 2, d // 2).transpose(3, 4)
        z = torch.view_as_real(torch.view_as_complex(z.contiguous()) * unit)
        return (z if inter else z.transpose(3, 4)).reshape(B, H, N, d)

    out = {}
    for i, name in enumerate(("q", "k")):
        x = s[name].double()
        w = s[name + "w"].double() if case["norm"] != "none" else None
        if case["kind"] == "rope":
            out[name] = one(x, w)
            continue
        leaves = [t.requires_grad_() for t in (x, w) if t is not None]
        grads = torch.autograd.grad(one(x, w), leaves, s["dout"][i].double())
        out["d" + name] = grads[0]
        if w is not None:
            out["d" + name + "w"] = grads[1]
    return out


def _exact_norm(s):
    case, part = s["case"], s["case"]["part"]
    before, after, bwd = part != "after", part != "before", case["kind"] == "norm_bwd"

    def norm(kind, t, w):
        if kind == "layer":
            t = (t - t.mean(-1, keepdim=True)) / (t.var(-1, unbiased=False, keepdim=True) + EPS).sqrt()
        elif kind == "rms":
            t = t / (t.pow(2).sum(-1, keepdim=True) / case["C"] + EPS).sqrt()
        return t if w is None else t * w

    def wide(m):
        return {"batch": lambda: m.unsqueeze(1), "token": lambda: m, "shared": lambda: m.view(1, 1, -1)}[case["mods"]]()

    p = {k: s[k].double() for k in ("gate", "scale", "shift")}
    wi = s["wi"].double() if case["weights"] and before else None
    wo = s["wo"].double() if case["weights"] and after and case["norm_out"] != "none" else None
    if not bwd:
        out, x = {}, s["x"].double()
        if after:
            x = case["rho"] * x + wide(p["gate"]) * norm(case["norm_out"], s["y"].double(), wo)
            out["x_out"] = x
            x = x.to(s["x"].dtype).double()                       # h is taken of what is stored
        if before:
            out["h"] = norm(case["norm_in"], x, wi) * (1 + wide(p["scale"])) + wide(p["shift"])
        return out
    out, u = {}, s["dx_out"].double()
    if before:
        x = s["x"].double()
        leaves = {"x": x, "dscale": p["scale"], "dshift": p["shift"]}
        if wi is not None:
            leaves["dwi"] = wi
        names = list(leaves)
        h = norm(case["norm_in"], x.requires_grad_(), wi.requires_grad_() if wi is not None else None)
        h = h * (1 + wide(p["scale"].requires_grad_())) + wide(p["shift"].requires_grad_())
        got = dict(zip(names, torch.autograd.grad(h, [leaves[k] for k in names], s["dh"].double())))
        u = u + got.pop("x")
        out.update(got)
    if after:
        y = s["y"].double()
        leaves = {"dy": y, "dgate": p["gate"]}
        if wo is not None:
            leaves["dwo"] = wo
        names = list(leaves)
        m = wide(p["gate"].requires_grad_()) * norm(case["norm_out"], y.requires_grad_(), wo.requires_grad_() if wo is not None else None)
        out.update(zip(names, torch.autograd.grad(m, [leaves[k] for k in names], u)))
        u = case["rho"] * u
    out["dx"] = u
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return (_exact_rope if case["kind"].startswith("rope") else _exact_norm)(s)
