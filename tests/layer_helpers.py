"""Shared plumbing of the tests of sla2_rope_* and sla2_norm_*: tensors of a layout, error bounds.

Bounds.  The library rounds once to the stored type (off by half a step, finfo.eps / 2 of the value) what fp32 arithmetic made.  The
latter's error is counted in units of 2^-24 of `mag`, the sum of the absolute values of a result's terms.  A row's sum has at most 16
terms in turn in a lane, 6 steps over the lanes and 8 over the waves: below 32 roundings, its mean and root below 8 more; a result has
fewer than 24 roundings of its own (products, sums, the angle, cos and sin of 2 steps each).  So 64 units cover a value of a row, and
gradients summed over rows have, on top, one rounding per row that a lane adds and below 64 for the joining of teams and workgroups."""
import numpy as np

UNIT = 2.0 ** -24
ROW_UNITS = 64
# bf16 tensors: cos and sin are the hardware's, taken to be good to 2^-17 of a turn's radius - 512 times finer than half a step of bf16
TRIG_UNITS = 128


def close(got, ref, mag, dtype, units=ROW_UNITS, what=""):
    """got: torch tensor; ref, mag: fp64 arrays."""
    import torch
    g = got.detach().double().cpu().numpy()
    assert g.shape == ref.shape, (what, g.shape, ref.shape)
    half = torch.finfo(dtype).eps / 2
    bound = half * np.abs(ref) + units * UNIT * (1 + half) * np.broadcast_to(mag, ref.shape) + torch.finfo(dtype).smallest_normal
    bad = ~(np.abs(g - ref) <= bound)                 # a NaN is bad
    assert not bad.any(), "%s: %d of %d out of bounds, worst %g times" % (
        what, int(bad.sum()), bad.size, float(np.nanmax(np.abs(g - ref) / bound)))


def f64(t):
    return t.detach().double().cpu().numpy()


def sum_units(rows):
    """For gradients summed over `rows` rows of which a lane adds at most that many, one after the other."""
    return 2 * ROW_UNITS + rows


PAD = 8                                               # elements between rows that must be left alone
GUARD = 7.0


def heads_like(torch, B, H, N, d, layout, dtype, gen=None, n=2):
    """n tensors [B, H, N, d] (views), the (batch, head, token) strides that they share, and the buffers they lie in."""
    if layout == "packed":
        buf = torch.full((B, N, n + 1, H, d), GUARD, dtype=dtype, device="cuda")
        ts = [buf[:, :, i].permute(0, 2, 1, 3) for i in range(n)]
        st, bufs = (N * (n + 1) * H * d, d, (n + 1) * H * d), [buf]
    elif layout == "padded":
        bufs = [torch.full((B, N, H, d + PAD), GUARD, dtype=dtype, device="cuda") for _ in range(n)]
        ts = [b[..., :d].permute(0, 2, 1, 3) for b in bufs]
        st = (N * H * (d + PAD), d + PAD, H * (d + PAD))
    elif layout == "tokens":
        bufs = [torch.full((B, N, H, d), GUARD, dtype=dtype, device="cuda") for _ in range(n)]
        ts = [b.permute(0, 2, 1, 3) for b in bufs]
        st = (N * H * d, d, H * d)
    else:
        bufs = [torch.full((B, H, N, d), GUARD, dtype=dtype, device="cuda") for _ in range(n)]
        ts, st = bufs, None
    if gen is not None:
        for t in ts:
            t.copy_(torch.randn((B, H, N, d), generator=gen, device="cuda"))
    return ts, st, bufs


def guards_ok(layout, bufs, n=2):
    for b in bufs:
        if layout == "packed":
            assert bool((b[:, :, n] == GUARD).all())
        elif layout == "padded":
            assert bool((b[..., -PAD:] == GUARD).all())
