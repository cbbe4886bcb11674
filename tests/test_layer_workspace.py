"""The workspace of sla2_rope_backward and sla2_norm_backward among the tensors of the call: partial sums written over one of them would be
wrong gradients without an error.  Every call below is refused before a device is touched."""
import pytest

import test_layer_abi as T
from paper_2602_12675_amd import api

EALIAS, EWORKSPACE = api.SLA2_EALIAS, api.SLA2_EWORKSPACE


@pytest.mark.parametrize("norm", [api.SLA2_ROPE_NORM_HEAD, api.SLA2_ROPE_NORM_TOKEN])
@pytest.mark.parametrize("where", ["q", "k", "freq", "positions", "q_weight", "k_weight", "dq_out", "dk_out", "dq", "dk", "dq_weight", "dk_weight"])
def test_rope(where, norm):
    at = dict(q=T.Q, k=T.K, freq=T.FREQ, positions=T.POS, q_weight=T.QW, k_weight=T.KW, dq_out=T.QO, dk_out=T.KO, dq=T.DQ, dk=T.DK,
              dq_weight=T.DQW, dk_weight=T.DKW)[where]
    p = T.rope(norm=norm)
    need = api.sla2_rope_workspace_bytes(p)
    size = {"freq": 32 * 8, "positions": 10 * 3 * 4}.get(where, (64 if norm == api.SLA2_ROPE_NORM_HEAD else 192) * 4 if "weight" in where
                                                       else 2 * 3 * 10 * 64 * 2)
    assert T.rope_backward(p, workspace=at, ws_bytes=need) == EALIAS
    assert T.rope_backward(p, workspace=at + (size - 16) // 256 * 256, ws_bytes=need) == EALIAS            # its first bytes on the tensor's last
    assert T.rope_backward(p, workspace=at - need + 256, ws_bytes=need) == EALIAS                          # its last ones on the tensor's first
    if "weight" not in where:                                                                              # one gradient wanted, either of them
        assert T.rope_backward(p, workspace=at, dq_weight=None) == EALIAS and T.rope_backward(p, workspace=at, dk_weight=None) == EALIAS


@pytest.mark.parametrize("mods", [api.SLA2_MOD_BATCH, api.SLA2_MOD_TOKEN, api.SLA2_MOD_SHARED])
@pytest.mark.parametrize("where", ["x", "y", "gate", "out_weight", "in_weight", "scale", "dh", "dx_out", "dx", "dy", "dgate", "dout_weight",
                                   "din_weight", "dscale", "dshift"])
def test_norm(where, mods):
    at = dict(x=T.X, y=T.Y, gate=T.GATE, out_weight=T.OW, in_weight=T.IW, scale=T.SCALE, dh=T.DH, dx_out=T.DXO, dx=T.DX, dy=T.DY, dgate=T.DG,
              dout_weight=T.DOW, din_weight=T.DIW, dscale=T.DS, dshift=T.DB)[where]
    p = T.norm(mod_layout=mods)
    need = api.sla2_norm_workspace_bytes(p)
    assert T.norm_backward(p, workspace=at, ws_bytes=need) == EALIAS
    assert T.norm_backward(p, workspace=at - need + 256, ws_bytes=need) == EALIAS
    if where in ("x", "y", "dh", "dx_out", "dx", "dy"):
        last = 2 * 10 * 64 * (4 if where in ("x", "dx", "dx_out") else 2) - 256
        assert T.norm_backward(p, workspace=at + last, ws_bytes=need) == EALIAS


def test_beside_the_tensors_it_is_not_refused_as_an_alias():
    """Right behind or before a tensor: what is refused here is its size, which is looked at last."""
    p = T.rope()
    need, size = api.sla2_rope_workspace_bytes(p), 2 * 3 * 10 * 64 * 2
    assert T.rope_backward(p, workspace=T.DK + size, ws_bytes=need - 256) == EWORKSPACE
    assert T.rope_backward(p, workspace=T.DK - need, ws_bytes=need - 256) == EWORKSPACE
    p = T.norm()
    need = api.sla2_norm_workspace_bytes(p)
    assert T.norm_backward(p, workspace=T.DX + 2 * 10 * 64 * 4, ws_bytes=need - 256) == EWORKSPACE
    assert T.norm_backward(p, workspace=T.DX - need, ws_bytes=need - 256) == EWORKSPACE
