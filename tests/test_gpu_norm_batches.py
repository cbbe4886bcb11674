"""sla2_norm_backward over many sequences: more columns of gradients than one launch has threads for."""
import pytest

from layer_helpers import UNIT

pytestmark = pytest.mark.gpu


def test_more_sums_of_columns_than_a_launch_has_threads():
    """10,930 sequences of one token of 8,192 channels, gate, scale and shift of each: 256 tiles of columns x (3 x 10,930 + 2) sums, of 512 threads
    each, are more than 2^32 threads.  Sequences share nothing but the weights, so the halves of the batch in calls of their own give the
    same bits; the weights' gradients are sums of what the sequences' are."""
    import torch
    from paper_2602_12675_amd import api
    B, C = 10930, 8192
    assert (C // 32) * (3 * B + 2) * 512 >= 2 ** 32 and (C // 32) * (3 * (B // 2) + 2) * 512 < 2 ** 32
    gen = torch.Generator(device="cuda").manual_seed(5)
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda", dtype=torch.bfloat16)                       # noqa: E731
    x, y, dh, dx_out = (rand(B, 1, C) for _ in range(4))
    gate, scale = (rand(B, C).float() for _ in range(2))
    one = torch.ones(C, device="cuda")

    def run(at):
        n = at.stop - at.start
        p = api.make_norm_params(n, 1, C, norm_in=api.SLA2_NORM_LAYER, norm_out=api.SLA2_NORM_RMS)
        out = {k: torch.full((n, C), 7.0, device="cuda") for k in ("dgate", "dscale", "dshift")}
        out.update({k: torch.full((C,), 7.0, device="cuda") for k in ("dout_weight", "din_weight")})
        dx, dy = torch.empty_like(x[at]), torch.empty_like(y[at])
        ws = torch.empty(api.sla2_norm_workspace_bytes(p), dtype=torch.uint8, device="cuda")
        api.sla2_norm_backward(p, x[at], dh[at], dx_out[at], dx, y=y[at], gate=gate[at], out_weight=one, in_weight=one, scale=scale[at],
                               dy=dy, workspace=ws, **out)
        return dict(out, dx=dx, dy=dy)

    whole = run(slice(0, B))
    for at in (slice(0, B // 2), slice(B // 2, B)):
        for name, t in run(at).items():
            if "weight" not in name:
                assert torch.equal(whole[name][at], t), (name, at)
    # each term is rounded with 1 + s and with the product; a lane adds ceil(B / 64) of them in turn, then 6 halves of 64 lanes
    units = 2 + -(-B // 64) + 6
    for name, of, m in (("din_weight", "dscale", 1 + scale), ("dout_weight", "dgate", gate)):
        want, mag = torch.zeros(C, dtype=torch.float64, device="cuda"), torch.zeros(C, dtype=torch.float64, device="cuda")
        for at in range(0, B, 1024):
            terms = whole[of][at:at + 1024].double() * m[at:at + 1024].double()
            want += terms.sum(0)
            mag += terms.abs().sum(0)
        assert bool(((whole[name].double() - want).abs() <= units * UNIT * mag).all()), name
