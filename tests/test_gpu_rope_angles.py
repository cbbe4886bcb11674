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
    """`units` steps of 2^-24 of the value; and of the angle, in fp64: the products with the frequency, with 1 / 2 pi (which is rounded
    too) and the reference's.

    3 units are what cosine and sine are off by.  With |x| <= pi / 4 rounded to fp32 once: the sine 1 for x, 1 for the last sum, and 0.1 (x^2 / 6) of
    the 3 roundings that its square and the series have had; the cosine 0.8 (x tan x) for x, 0.7 for the last sum (half a step below 1, of
    0.71), and 0.44 (x^2 / 2 of 0.71) of the 3 others."""
    return units * UNIT * np.abs(ref) + 5 * 2.0 ** -53 * np.abs(angle)


@pytest.mark.parametrize("halves", [False, True], ids=["pairs", "halves"])
@pytest.mark.parametrize("d,axes", [(64, (8, 12, 12)), (128, (22, 21, 21))])
def test_cosine_and_sine_of_fp32_results(d, axes, halves):
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
            bad = ~(np.abs(value - ref) <= trig_bound(ref, angle, 3))         # a NaN is bad
            assert not bad.any(), (value[bad][:4], ref[bad][:4])


@pytest.mark.parametrize("halves", [False, True], ids=["pairs", "halves"])
@pytest.mark.parametrize("norm", ["head", "token"])
@pytest.mark.parametrize("d,axes,H,N", [(64, (8, 12, 12), 1, 1), (128, (22, 21, 21), 1, 1), (128, (64, 0, 0), 1, 5), (64, (0, 16, 16), 3, 700)])
def test_gradients_of_the_weights_of_bf16_tensors(d, axes, H, N, norm, halves):
    """They are fp32 whatever the tensors are.  x = 1 and dy = (1, 0) at one token, 0 at the others: dw is r cos and -r sin of that
    token's angles, and every other term is an exact 0.  8 units: 3 of cosine and sine, 2 of the root (a step of 2^-23), half of the sum with
    eps, 1 each of the product of x with the root and with g.  The sum of the squares and its mean are exact; eps leaves r at
    1 / sqrt(1 + eps), which the reference has."""
    import torch
    from paper_2602_12675_amd import api
    rng = np.random.default_rng(d + N + halves)
    eps = 1e-5
    p = api.make_rope_params(1, H, N, d, axes, dtype=api.SLA2_BF16, pairing=int(halves), eps=eps,
                             norm={"head": api.SLA2_ROPE_NORM_HEAD, "token": api.SLA2_ROPE_NORM_TOKEN}[norm])
    x = torch.ones((1, H, N, d), dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(api.sla2_rope_workspace_bytes(p), dtype=torch.uint8, device="cuda")
    shape = (H, d) if norm == "token" else (d,)
    for _ in range(20):
        positions, freq = rng.integers(-3000, 3000, (N, 3)).astype(np.int32), rng.uniform(0.01, 3.0, d // 2)
        n, h = int(rng.integers(N)), int(rng.integers(H))
        g = torch.zeros_like(x)
        g[0, h, n] = ones_and_zeros(torch, 1, d, halves, torch.bfloat16)[0, 0, 0]
        dx, dw = torch.empty_like(x), torch.full(shape, 7.0, device="cuda")
        api.sla2_rope_backward(p, x, None, torch.from_numpy(freq).cuda(), g, None, dx, None, dq_weight=dw,
                               positions=torch.from_numpy(positions).cuda(), workspace=ws)
        dw = f64(dw)
        if norm == "token":
            assert not dw[np.arange(H) != h].any()
            dw = dw[h]
        angle = angles(positions[n:n + 1], freq, axes)[0]
        c, s = split(dw, halves)
        r = 1.0 / np.sqrt(1.0 + float(np.float32(eps)))
        for value, ref in ((c, r * np.cos(angle)), (s, -r * np.sin(angle))):
            bad = ~(np.abs(value - ref) <= trig_bound(ref, angle, 8))
            assert not bad.any(), (value[bad][:4], ref[bad][:4])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_angles_without_a_fraction_are_rotations_still(dtype):
    """Angles of 2^53 turns and more, of which fp64 holds no fraction: whatever they are, cos^2 + sin^2 is 1 (each is off by half a step of its
    type at most, of bf16 2^-8, and by 3 units of 2^-24)."""
    import torch
    from paper_2602_12675_amd import api
    N, d, ty = 40, 64, {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    rng = np.random.default_rng(1)
    p = api.make_rope_params(1, 1, N, d, (32, 0, 0), dtype=api.SLA2_F32 if dtype == "f32" else api.SLA2_BF16, norm=api.SLA2_ROPE_NORM_HEAD)
    freq = torch.from_numpy(10.0 ** rng.uniform(10, 60, d // 2)).cuda()
    at = torch.from_numpy(rng.integers(2 ** 30, 2 ** 31, (N, 3)).astype(np.int32)).cuda()
    x = ones_and_zeros(torch, N, d, False, ty)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    plain = api.make_rope_params(1, 1, N, d, (32, 0, 0), dtype=p.dtype)
    half = torch.finfo(ty).eps / 2
    api.sla2_rope_forward(plain, x, None, freq, y, None, positions=at)
    api.sla2_rope_backward(plain, None, None, freq, x, None, dx, None, positions=at)
    for t in (y, dx):
        c, s = split(f64(t)[0, 0], False)
        assert np.abs(c * c + s * s - 1).max() <= 2 * (half + 3 * UNIT) * (1 + half)
    # dy = x: n = sqrt(2) (1, 0), so dw = sqrt(2) cos at the channels of x and 0 at the others, token by token
    ws = torch.empty(api.sla2_rope_workspace_bytes(p), dtype=torch.uint8, device="cuda")
    dw = torch.empty(d, device="cuda")
    api.sla2_rope_backward(p, x, None, freq, x, None, dx, None, dq_weight=dw, positions=at, workspace=ws)
    c, s = split(f64(dw)[None], False)
    assert not s.any() and np.abs(c).max() <= N * np.sqrt(2) * (1 + 1e-5)
