"""Host-side checks of sla2_rope_* and sla2_norm_*: the structures, the frequencies, and the refusal of bad arguments before a
device is touched.  No compute call is made here (no GPU needed): every call below is refused."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

import layer_oracle as L
from paper_2602_12675_amd import api

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EINVAL, EUNSUPPORTED, EWORKSPACE, EALIAS = api.SLA2_EINVAL, api.SLA2_EUNSUPPORTED, api.SLA2_EWORKSPACE, api.SLA2_EALIAS

_PROBE = r"""
#include <stdio.h>
#include <stddef.h>
#include "sla2.h"
int main(void) {
@BODY@
  return 0;
}
"""


def test_structures_match_the_header(tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("no C compiler")
    lines, want = [], []
    for cname, cls in (("sla2_rope_params", api.RopeParams), ("sla2_norm_params", api.NormParams)):
        lines.append('  printf("%%zu\\n", sizeof(%s));' % cname)
        want.append(ctypes.sizeof(cls))
        for name, _ in cls._fields_:
            lines.append('  printf("%%zu\\n%%zu\\n", offsetof(%s, %s), sizeof(((%s*)0)->%s));' % (cname, name, cname, name))
            want += [getattr(cls, name).offset, getattr(cls, name).size]
    src, exe = tmp_path / "p.c", tmp_path / "p"
    src.write_text(_PROBE.replace("@BODY@", "\n".join(lines)))
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-pedantic", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    assert got == want


def test_frequencies():
    for d, axes, theta in ((128, (22, 21, 21), 10000.0), (64, (0, 16, 16), 256.0), (64, (32, 0, 0), 1e6), (128, (3, 0, 5), 7.0), (64, (0, 0, 0), 2.0)):
        f = api.sla2_rope_frequencies(api.make_rope_params(1, 1, 1, d, axes), theta)
        assert f.dtype == torch.float64 and f.shape == (d // 2,)
        np.testing.assert_allclose(f.numpy(), L.frequencies(axes, d, theta), rtol=1e-14, atol=0)
    for theta in (0.0, -1.0, float("nan"), float("inf")):
        with pytest.raises(api.Sla2Error):
            api.sla2_rope_frequencies(api.make_rope_params(1, 1, 1, 64, (32, 0, 0)), theta)


# ---- rope ----
def rope(**kw):
    base = dict(B=2, H=3, N=10, d=64, axis_pairs=(10, 11, 11), norm=api.SLA2_ROPE_NORM_TOKEN)
    base.update(kw)
    return api.make_rope_params(**base)


Q, K, QO, KO, FREQ, POS, QW, KW, DQ, DK, DQW, DKW, WS = (i << 20 for i in range(1, 14))


def rope_forward(p, q=Q, k=K, freq=FREQ, q_out=QO, k_out=KO, **kw):
    kw = dict(dict(q_weight=QW, k_weight=KW, positions=POS), **kw)
    return api.sla2_rope_forward(p, q, k, freq, q_out, k_out, check=False, **kw)


def rope_backward(p, q=Q, k=K, freq=FREQ, dq_out=QO, dk_out=KO, dq=DQ, dk=DK, ws_bytes=1 << 19, **kw):
    kw = dict(dict(q_weight=QW, k_weight=KW, dq_weight=DQW, dk_weight=DKW, positions=POS, workspace=WS), **kw)
    return api.sla2_rope_backward(p, q, k, freq, dq_out, dk_out, dq, dk, ws_bytes=ws_bytes, check=False, **kw)


@pytest.mark.parametrize("kw,status", [
    (dict(B=0), EINVAL), (dict(H=-1), EINVAL), (dict(N=0), EINVAL), (dict(d=96), EUNSUPPORTED), (dict(d=0), EUNSUPPORTED),
    (dict(dtype=2), EINVAL), (dict(pairing=2), EINVAL), (dict(norm=3), EINVAL), (dict(norm=-1), EINVAL),
    (dict(eps=0.0), EINVAL), (dict(eps=float("nan")), EINVAL), (dict(eps=float("inf")), EINVAL), (dict(positions_per_batch=2), EINVAL),
    (dict(eps=1e-39), EINVAL), (dict(eps=-1e-6), EINVAL),
    (dict(axis_pairs=(11, 11, 11)), EINVAL), (dict(axis_pairs=(-1, 11, 11)), EINVAL), (dict(axis_pairs=(2 ** 31 - 1, 2 ** 31 - 1, 2)), EINVAL),
    (dict(grid=(0, 2, 5)), EINVAL), (dict(grid=(2, -1, 5)), EINVAL), (dict(grid=(2 ** 16, 2 ** 15, 1)), EUNSUPPORTED),
    (dict(grid=(2, 1, 5), origin=(2 ** 31 - 1, 0, 0)), EINVAL), (dict(origin=(1, 0, 0)), EINVAL),
    (dict(B=256, H=256), EUNSUPPORTED), (dict(H=129), EUNSUPPORTED),
    (dict(in_stride=(0, 64, 64)), EINVAL), (dict(out_stride=(-64, 64, 64)), EINVAL), (dict(in_stride=(1920, 640, 32)), EUNSUPPORTED),
    (dict(out_stride=(1920, 644, 64)), EUNSUPPORTED), (dict(in_stride=(1 << 60, 64, 192)), EUNSUPPORTED),
])
def test_bad_rope_parameters(kw, status):
    p = rope(**kw)
    assert api.sla2_rope_workspace_bytes(p) == 0
    assert rope_forward(p, positions=None if "grid" in kw else POS) == status
    assert rope_backward(p, positions=None if "grid" in kw else POS) == status
    with pytest.raises(api.Sla2Error):
        api.sla2_rope_frequencies(p)


def test_bad_rope_pointers():
    p, grid, plain = rope(), rope(grid=(1, 2, 5)), rope(norm=api.SLA2_ROPE_NORM_NONE)
    for kw in (dict(q=None), dict(q_out=None), dict(k=None), dict(k_out=None), dict(freq=None), dict(positions=None), dict(q=Q + 8),
               dict(k=K + 2), dict(q_out=QO + 4), dict(k_out=KO + 8), dict(freq=FREQ + 4), dict(positions=POS + 2), dict(q_weight=QW + 4),
               dict(k_weight=KW + 8), dict(k=None, k_out=None)):
        assert rope_forward(p, **kw) == EINVAL, kw                 # the last: a weight of k without k
    assert rope_forward(grid) == EINVAL                            # a grid and positions
    assert rope_forward(plain) == EINVAL                           # weights without a norm
    for kw in (dict(q=None), dict(k=None), dict(dq_out=None), dict(dk_out=None), dict(dq=None), dict(dk=None), dict(freq=None),
               dict(positions=None), dict(dq=DQ + 8), dict(dk_out=KO + 8), dict(dq_weight=DQW + 4), dict(dk_weight=DKW + 8),
               dict(k=None, dk=None, dk_out=None), dict(k=None, dk=None, dk_out=None, k_weight=None)):
        assert rope_backward(p, **kw) == EINVAL, kw
    assert rope_backward(plain, q_weight=None, k_weight=None) == EINVAL          # gradients of weights that are not there
    need = api.sla2_rope_workspace_bytes(p)
    assert need > 0
    for kw in (dict(workspace=None), dict(workspace=WS + 16), dict(ws_bytes=need // 2), dict(ws_bytes=0)):
        assert rope_backward(p, **kw) == EWORKSPACE, kw
    assert api.sla2_rope_workspace_bytes(plain) > 0                # not the 0 of invalid parameters


def test_rope_aliases():
    size = 2 * 3 * 10 * 64 * 2
    p = rope()
    for kw in (dict(q_out=K), dict(k_out=Q), dict(q_out=Q + 16), dict(q_out=Q + size - 16), dict(k_out=QO), dict(k_out=QO + size - 16),
               dict(q_out=FREQ - 16), dict(k_out=POS), dict(q_out=QW - size + 16), dict(k_out=KW)):
        assert rope_forward(p, **kw) == EALIAS, kw
    # in place takes one layout
    assert rope_forward(rope(out_stride=(3 * 640, 640, 64), in_stride=(3 * 640, 64, 192)), q_out=Q) == EALIAS
    # slices of one packed buffer, a row apart: disjoint; half a row apart: not
    st = (10 * 3 * 192, 64, 3 * 192)
    packed = rope(in_stride=st, out_stride=st)
    assert rope_forward(packed, q=Q, k=Q + 384, q_out=Q + 192, k_out=Q + 768) == EALIAS
    assert rope_forward(packed, q=Q, k=Q + 384, q_out=Q, k_out=Q) == EALIAS
    assert rope_backward(packed, dq=DQ, dk=DQ + 192) == EALIAS
    assert rope_backward(packed, q=Q, k=Q + 384, dq=Q + 384, dk=Q) == EALIAS     # each on the other's input
    for kw in (dict(dq=K), dict(dk=KO - 16), dict(dq=DK), dict(dq_weight=DKW), dict(dk_weight=DQ), dict(dq_weight=QW), dict(dq_weight=Q)):
        assert rope_backward(p, **kw) == EALIAS, kw


# ---- norm ----
X, Y, GATE, OW, XO, IW, SCALE, SHIFT, H_, DH, DXO, DX, DY, DG, DOW, DIW, DS, DB, NWS = (i << 20 for i in range(1, 20))


def norm(**kw):
    base = dict(B=2, N=10, C=64, dtype_x=api.SLA2_F32, dtype_h=api.SLA2_BF16, norm_in=api.SLA2_NORM_LAYER, norm_out=api.SLA2_NORM_RMS)
    base.update(kw)
    return api.make_norm_params(**base)


def norm_forward(p, x=X, h=H_, **kw):
    kw = dict(dict(y=Y, x_out=XO, gate=GATE, out_weight=OW, in_weight=IW, scale=SCALE, shift=SHIFT), **kw)
    return api.sla2_norm_forward(p, x, h, check=False, **kw)


def norm_backward(p, x=X, dh=DH, dx_out=DXO, dx=DX, ws_bytes=1 << 19, **kw):
    kw = dict(dict(y=Y, gate=GATE, out_weight=OW, in_weight=IW, scale=SCALE, dy=DY, dgate=DG, dout_weight=DOW, din_weight=DIW, dscale=DS,
                   dshift=DB, workspace=NWS), **kw)
    return api.sla2_norm_backward(p, x, dh, dx_out, dx, ws_bytes=ws_bytes, check=False, **kw)


@pytest.mark.parametrize("kw,status", [
    (dict(B=0), EINVAL), (dict(N=0), EINVAL), (dict(C=0), EINVAL), (dict(C=-8), EINVAL), (dict(C=100), EUNSUPPORTED),
    (dict(C=8200), EUNSUPPORTED), (dict(B=65536), EUNSUPPORTED), (dict(dtype_x=2), EINVAL), (dict(dtype_h=-1), EINVAL),
    (dict(dtype_x=1, dtype_h=0), EUNSUPPORTED), (dict(norm_in=3), EINVAL), (dict(norm_out=-1), EINVAL), (dict(eps=0.0), EINVAL),
    (dict(eps=float("nan")), EINVAL), (dict(eps=float("inf")), EINVAL), (dict(residual_scale=float("nan")), EINVAL), (dict(eps=1e-39), EINVAL),
    (dict(residual_scale=float("inf")), EINVAL), (dict(mod_layout=3), EINVAL), (dict(x_stride=(0, 64)), EINVAL),
    (dict(x_stride=(640, -64)), EINVAL), (dict(x_stride=(640, 60)), EUNSUPPORTED), (dict(h_stride=(640, 68)), EUNSUPPORTED),
    (dict(h_stride=(644, 64)), EUNSUPPORTED), (dict(x_stride=(1 << 60, 64)), EUNSUPPORTED), (dict(mod_stride=(64, 64)), EINVAL),
    (dict(mod_stride=(60, 0)), EUNSUPPORTED), (dict(mod_stride=(66, 0)), EUNSUPPORTED), (dict(mod_stride=(-64, 0)), EINVAL),
    (dict(mod_layout=1, mod_stride=(640, 0)), EINVAL), (dict(mod_layout=1, mod_stride=(0, 64)), EINVAL),
    (dict(mod_layout=1, mod_stride=(640, 60)), EUNSUPPORTED), (dict(mod_layout=2, mod_stride=(64, 0)), EINVAL),
])
def test_bad_norm_parameters(kw, status):
    p = norm(**kw)
    assert api.sla2_norm_workspace_bytes(p) == 0
    assert norm_forward(p) == status
    assert norm_backward(p) == status


def test_bad_norm_pointers():
    p = norm()
    none_after = dict(y=None, x_out=None, gate=None, out_weight=None)
    none_before = dict(h=None, in_weight=None, scale=None, shift=None)
    for kw in (dict(x=None), dict(y=None), dict(x_out=None), dict(none_after, gate=GATE), dict(none_after, out_weight=OW),
               dict(none_after, x_out=XO), dict(none_before, scale=SCALE), dict(none_before, shift=SHIFT), dict(none_before, in_weight=IW),
               dict(none_after, **none_before), dict(x=X + 4), dict(y=Y + 8), dict(x_out=XO + 2), dict(h=H_ + 8), dict(gate=GATE + 4),
               dict(out_weight=OW + 8), dict(in_weight=IW + 4), dict(scale=SCALE + 4), dict(shift=SHIFT + 12)):
        assert norm_forward(p, **kw) == EINVAL, kw
    after = dict(y=None, dy=None, gate=None, out_weight=None, dgate=None, dout_weight=None)
    before = dict(dh=None, in_weight=None, scale=None, din_weight=None, dscale=None, dshift=None)
    for kw in (dict(dx=None), dict(y=None), dict(dy=None), dict(x=None), dict(after, gate=GATE), dict(after, dgate=DG), dict(after, out_weight=OW),
               dict(before, scale=SCALE), dict(before, dshift=DB), dict(before, in_weight=IW), dict(before, dx_out=None), dict(after, **before),
               dict(gate=None), dict(scale=None), dict(in_weight=None), dict(out_weight=None), dict(dx=DX + 4), dict(dy=DY + 8),
               dict(dh=DH + 2), dict(dx_out=DXO + 8), dict(dgate=DG + 4), dict(dscale=DS + 4), dict(dshift=DB + 8), dict(din_weight=DIW + 4),
               dict(dout_weight=DOW + 4)):
        assert norm_backward(p, **kw) == EINVAL, kw
    need = api.sla2_norm_workspace_bytes(p)
    assert need > 0
    for kw in (dict(workspace=None), dict(workspace=NWS + 128), dict(ws_bytes=need // 2)):
        assert norm_backward(p, **kw) == EWORKSPACE, kw
    for name in ("dgate", "dout_weight", "din_weight", "dscale", "dshift"):                # any one of them takes the workspace
        rest = {n: None for n in ("dgate", "dout_weight", "din_weight", "dscale", "dshift") if n != name}
        assert norm_backward(p, workspace=None, **rest) == EWORKSPACE, name


def test_norm_aliases():
    p, size = norm(), 2 * 10 * 64
    for kw in (dict(x_out=X + 16), dict(x_out=X + 4 * size - 16), dict(h=Y + 16), dict(h=X), dict(x_out=Y), dict(h=XO), dict(x_out=GATE),
               dict(h=SHIFT - 16), dict(x_out=IW), dict(h=OW)):
        assert norm_forward(p, **kw) == EALIAS, kw
    for kw in (dict(dx=X + 16), dict(dx=DY), dict(dy=X), dict(dy=DXO), dict(dx=DXO + 16), dict(dgate=GATE), dict(dscale=DS, dshift=DS),
               dict(dgate=DX), dict(din_weight=DOW), dict(din_weight=IW), dict(dshift=DH)):
        assert norm_backward(p, **kw) == EALIAS, kw
    # the gradients of the modulation as slices of one [B, 6, C] buffer are apart; half a slice further they are not
    six = norm(mod_stride=(6 * 64, 0))
    assert norm_backward(six, dgate=DG, dscale=DG + 256, dshift=DG + 384) == EALIAS


def test_a_view_without_stated_strides_is_refused():
    """An expanded or permuted tensor with the default layout would be read beyond its storage or in the wrong order."""
    class OnGpu(torch.Tensor):                                     # what the binding sees of a tensor on a GPU; never launched
        def get_device(self):
            return 0

    def t(x):
        return x.as_subclass(OnGpu)
    p, x, h = norm(), torch.zeros(2, 10, 64), torch.zeros(2, 10, 64, dtype=torch.bfloat16)
    for kw in (dict(x=x[:1].expand(2, 10, 64)), dict(h=h.transpose(0, 1).contiguous().transpose(0, 1)), dict(scale=torch.zeros(64).expand(2, 64)),
               dict(shift=torch.zeros(2, 6, 64)[:, 1])):
        kw = {k: t(v) for k, v in dict(dict(x=x, h=h), **kw).items()}
        assert api.sla2_norm_forward(p, kw.pop("x"), kw.pop("h"), check=False, **kw) == EINVAL
    p, q = rope(norm=api.SLA2_ROPE_NORM_NONE, grid=(1, 2, 5)), torch.zeros(2, 10, 3, 3, 64, dtype=torch.bfloat16)
    f = t(torch.zeros(32, dtype=torch.float64))
    assert api.sla2_rope_forward(p, t(q[:, :, 0].transpose(1, 2)), None, f, t(q[:, :, 1].reshape(2, 3, 10, 64)), None, check=False) == EINVAL
    assert api.sla2_rope_forward(p, t(q[:, :, 0].reshape(2, 3, 10, 64)), None, f, t(q[:, :, 1]), None, check=False) == EINVAL


def test_the_binding_looks_at_tensors():
    """A tensor of another type, too small, or of vectors that are not contiguous: refused, never launched."""
    p = norm()
    x, h = torch.zeros(2, 10, 64), torch.zeros(2, 10, 64, dtype=torch.bfloat16)
    for bad in (dict(x=x.double()), dict(x=x[:, :9]), dict(h=x), dict(scale=torch.zeros(64)), dict(shift=torch.zeros(2, 64).double()),
                dict(in_weight=torch.zeros(128)[::2]), dict(in_weight=torch.zeros(63)), dict(y=h[:1], x_out=x)):
        kw = dict(dict(x=x, h=h), **bad)
        x_, h_ = kw.pop("x"), kw.pop("h")
        assert api.sla2_norm_forward(p, x_, h_, check=False, **kw) == EINVAL, bad
        with pytest.raises(api.Sla2Error):
            api.sla2_norm_forward(p, x_, h_, **kw)
    p = rope(norm=api.SLA2_ROPE_NORM_NONE)
    q, f, pos = torch.zeros(2, 3, 10, 64, dtype=torch.bfloat16), torch.zeros(32, dtype=torch.float64), torch.zeros(10, 3, dtype=torch.int32)
    for bad in (dict(q=q.float()), dict(freq=f.float()), dict(freq=f[:31]), dict(positions=pos.long()), dict(positions=pos[:9]),
                dict(positions=torch.zeros(3, 10, dtype=torch.int32).t()), dict(k=q, k_out=q[:1])):
        kw = dict(dict(q=q, k=None, freq=f, q_out=q.clone(), k_out=None, positions=pos), **bad)
        assert api.sla2_rope_forward(p, kw["q"], kw["k"], kw["freq"], kw["q_out"], kw["k_out"], positions=kw["positions"], check=False) == EINVAL, bad
