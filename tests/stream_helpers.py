"""Shared plumbing of the tests of sla2_packed_* and sla2_cache_*: inputs, layouts, error bounds.

Bounds.  A value is rounded to bf16 (off by half a step, 2^-8 of it) where it is stored, and P (times a value's scale) and dS are rounded
so on their way into the second product: 2^-8 of each term, which sums to at most 2^-8 of `mag`, the sum of the absolute values of a
result's terms.  fp32 arithmetic: a score is a sum of d products and the exponent's argument another 8 roundings (scale, reference,
exp2's 2 steps, sums' rescaling by powers that are rounded alike), each 2^-24 of at most `smag` = scale sum |q k| (and of the
reference, which is no larger; for the backward pass of |lse| too); a relative error of P is the absolute one of its exponent, times the
base's log2(e) < 1.5 and doubled for the sum of P that divides.  Sums over n terms: n roundings of 2^-24 of `mag`, however they are joined.
Numbers below 2^-126 may become 0: P and dS in front of their products, and results.  A term loses at most 2^-126 of its other factor."""
import numpy as np
import torch

UNIT = 2.0 ** -24
HALF = 2.0 ** -8                                      # bf16


def weight_error(d, n, smag):
    """Relative error of a probability and of a sum of n of them."""
    return UNIT * (3 * (d + 8) * smag + 2 * n + 32)


def close(got, ref, bound, what=""):
    g = got.detach().double().cpu().numpy() if hasattr(got, "detach") else np.asarray(got, dtype=np.float64)
    assert g.shape == ref.shape, (what, g.shape, ref.shape)
    same = (g == ref) | (np.abs(g - ref) <= bound)    # infinities are equal; a NaN is bad
    assert same.all(), "%s: %d of %d out of bounds, worst %g times, first at %s" % (
        what, int((~same).sum()), same.size, float(np.nanmax(np.abs(g - ref) / np.maximum(bound, 1e-300))), np.argwhere(~same)[0])


def out_bound(ref, mag, r):
    return HALF * np.abs(ref) + (HALF + r) * (1 + HALF) * mag + 2.0 ** -112   # n |v| up to 2^14, see tiny


def tiny(terms, factor):
    """What n terms that are 0 for less than 2^-126 may lose, and the result itself."""
    return 2.0 ** -126 * (1 + terms * float(np.abs(factor).max(initial=0.0)))


def lse_bound(lse, r):
    return np.where(np.isfinite(lse), r + 4 * UNIT * np.abs(np.where(np.isfinite(lse), lse, 0)), 0)


def starts(lengths, lead=0):
    return [lead + int(x) for x in np.concatenate([[0], np.cumsum(lengths)])]


def dev(x, dtype=torch.int32):
    return torch.tensor(x, dtype=dtype, device="cuda")


def f64(t):
    return t.detach().double().cpu().numpy()


PAD, GUARD = 8, 7.0


def rows_like(rows, heads, d, layout, gen=None, by=1.0):
    """A [rows, heads, d] tensor of bf16 (a view), its (head, token) strides or None, and the buffer."""
    if layout == "padded":                            # room behind every head and token
        buf = torch.full((rows, heads + 1, d + PAD), GUARD, dtype=torch.bfloat16, device="cuda")
        t, st = buf[:, :heads, :d], (d + PAD, (heads + 1) * (d + PAD))
    elif layout == "heads":                           # head-major
        buf = torch.full((heads, rows, d), GUARD, dtype=torch.bfloat16, device="cuda")
        t, st = buf.transpose(0, 1), (max(rows, 1) * d, d)
    else:
        buf = torch.full((rows, heads, d), GUARD, dtype=torch.bfloat16, device="cuda")
        t, st = buf, None
    if gen is not None and rows:
        t.copy_(by * torch.randn((rows, heads, d), generator=gen, device="cuda"))
    return t, st, buf


def guards_ok(layout, buf, heads, d):
    if layout == "padded":
        assert bool((buf[:, heads:] == GUARD).all()) and bool((buf[..., d:] == GUARD).all())
