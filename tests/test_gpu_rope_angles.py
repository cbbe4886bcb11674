"""The angles of sla2_rope_forward and sla2_rope_backward to the last bits: pairs of (1, 0), whose results are the cosine and the sine
themselves, so that an error of the angle shows where either is close to zero."""
import numpy as np
import pytest

from layer_helpers import UNIT, f64

pytestmark = pytest.mark.gpu


def angles(positions, freq, axes):
    """[N, d / 2] in fp64"""
    axis = np.repeat(np.arange(3), axes)
    return positions[:, axis].astype(np.float64) * freq


def ones_and_zeros(torch, N, d, halves, dtype):
    x = torch.zeros((1, 1, N, d), dtype=dtype, device="cuda")
    (x[..., :d // 2] if halves else x[..., 0::2]).fill_(1.0)
    return x


def split(x, halves):
    d = x.shape[-1]
    return (x[..., :d // 2], x[..., d // 2:]) if halves else (x[..., 0::2], x[..., 1::2])


def trig_bound(ref, angle, units):
    """`units` steps of 2^-24 of the value, and of the angle itself: the products with the frequency, with 1 / 2 pi (which is rounded too)
    and the reference's, in fp64; and 2^-45 for what is left of the rounding of the fraction of a turn: below 2^-23.3 it is added in fp32
    with three roundings and without its square (2^-23.3 x 3 x 2^-24 + 2^-47.6)."""
    return units * UNIT * np.abs(ref) + 2.0 ** -45 + 5 * 2.0 ** -53 * np.abs(angle)


@pytest.mark.parametrize("halves", [False, True], ids=["pairs", "halves"])
@pytest.mark.parametrize("d,axes", [(64, (8, 12, 12)), (128, (22, 21, 21))])
def test_cosine_and_sine_of_fp32_results(d, axes, halves):
    """5 units: 2 steps (of 2^-23) of the sine and cosine, half a step of the sum with what the fraction's rounding left."""
    import torch
    from paper_2602_12675_amd import api
    rng = np.random.default_rng(d + halves)
    N = 1500
    positions = rng.integers(-3000, 3000, (N, 3)).astype(np.int32)
    freq = rng.uniform(0.01, 3.0, d // 2)
    p = api.make_rope_params(1, 1, N, d, axes, dtype=api.SLA2_F32, pairing=int(halves))
    x = ones_and_zeros(torch, N, d, halves, torch.float32)
    y, back = torch.empty_like(x), torch.empty_like(x)
    at, f = torch.from_numpy(positions).cuda(), torch.from_numpy(freq).cuda()
    api.sla2_rope_forward(p, x, None, f, y, None, positions=at)
    api.sla2_rope_backward(p, None, None, f, x, None, back, None, positions=at)
    angle = angles(positions, freq, axes)
    for got, sign in ((y, 1.0), (back, -1.0)):
        c, s = split(f64(got)[0, 0], halves)
        for value, ref in ((c, np.cos(angle)), (s, sign * np.sin(angle))):
            error = np.abs(value - ref) / trig_bound(ref, angle, 5)
            assert error.max() <= 1.0, error.max()
