"""Host-side checks of sla2_packed_* and sla2_cache_*: the structures, the workspaces, and the refusal of bad arguments before a device
is touched.  No compute call is made here (no GPU needed): every call below is refused."""
import ctypes
import os
import shutil
import subprocess

import pytest
import torch

from paper_2602_12675_amd import api

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EINVAL, EUNSUPPORTED, EWORKSPACE, EALIAS = api.SLA2_EINVAL, api.SLA2_EUNSUPPORTED, api.SLA2_EWORKSPACE, api.SLA2_EALIAS
_PROBE = "#include <stdio.h>\n#include <stddef.h>\n#include \"sla2.h\"\nint main(void) {\n@BODY@\n  return 0;\n}\n"


def test_structures_match_the_header(tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("no C compiler")
    lines, want = [], []
    for cname, cls in (("sla2_packed_params", api.PackedParams), ("sla2_cache_params", api.CacheParams)):
        lines.append('  printf("%%zu\\n", sizeof(%s));' % cname)
        want.append(ctypes.sizeof(cls))
        for name, _ in cls._fields_:
            lines.append('  printf("%%zu\\n%%zu\\n", offsetof(%s, %s), sizeof(((%s*)0)->%s));' % (cname, name, cname, name))
            want += [getattr(cls, name).offset, getattr(cls, name).size]
    src, exe = tmp_path / "p.c", tmp_path / "p"
    src.write_text(_PROBE.replace("@BODY@", "\n".join(lines)))
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-pedantic", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    assert [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()] == want


# ---- packed ----
Q, K, V, QS, KS, OUT, LSE, DO, DQ, DK, DV, WS = (i << 20 for i in range(1, 13))
BIG = 1 << 19


def packed(**kw):
    return api.make_packed_params(**dict(dict(sequences=3, tokens_q=10, tokens_k=12, H=4, H_kv=2, d=64), **kw))


def forward(p, **kw):
    a = dict(dict(q=Q, k=K, v=V, q_start=QS, k_start=KS, out=OUT, lse=LSE, workspace=WS, ws_bytes=BIG), **kw)
    return api.sla2_packed_forward(p, check=False, **a)


def backward(p, **kw):
    a = dict(dict(q=Q, k=K, v=V, q_start=QS, k_start=KS, out=OUT, lse=LSE, dout=DO, dq=DQ, dk=DK, dv=DV, workspace=WS, ws_bytes=BIG), **kw)
    return api.sla2_packed_backward(p, check=False, **a)


@pytest.mark.parametrize("kw,status", [
    (dict(sequences=0), EINVAL), (dict(tokens_q=-1), EINVAL), (dict(tokens_k=-1), EINVAL), (dict(H=0), EINVAL), (dict(H_kv=0), EINVAL),
    (dict(H=3), EINVAL), (dict(d=96), EUNSUPPORTED), (dict(dtype=0), EUNSUPPORTED), (dict(dtype=2), EINVAL), (dict(causal=2), EINVAL),
    (dict(scale=-1.0), EINVAL), (dict(scale=float("nan")), EINVAL), (dict(scale=float("inf")), EINVAL), (dict(sequences=65536), EUNSUPPORTED),
    (dict(q_stride=(64, 0)), EINVAL), (dict(kv_stride=(-64, 128)), EINVAL), (dict(out_stride=(64, 260)), EUNSUPPORTED),
    (dict(q_stride=(68, 256)), EUNSUPPORTED), (dict(kv_stride=(64, 56)), EUNSUPPORTED), (dict(q_stride=(64, 1 << 24)), EUNSUPPORTED),
    (dict(q_stride=(1 << 60, 256)), EUNSUPPORTED), (dict(H=65536, H_kv=65536), EUNSUPPORTED),
    (dict(H=65535, H_kv=65535, tokens_q=2 ** 31 - 1), EUNSUPPORTED),
    (dict(sequences=65535, tokens_q=65535, tokens_k=65535, H=512, H_kv=512), EUNSUPPORTED),      # more workgroups than a launch may have
    (dict(tokens_k=2 ** 31 - 1, H=1, H_kv=1), EUNSUPPORTED),
])
def test_bad_packed_parameters(kw, status):
    p = packed(**kw)
    assert api.sla2_packed_workspace_bytes(p) == 0 and api.sla2_packed_workspace_bytes(p, True) == 0
    assert forward(p) == status and backward(p) == status


def test_parts_of_keys_have_a_bound():
    """Of many short sequences none has to be dealt to several workgroups, but one might be long: room for its parts, up to 1 GiB."""
    p = api.make_packed_params(1000, 200_000, 200_000, 64, 8, 128)
    n = 2 * (200_000 + 16 * 1000) * 64 * 4
    assert n <= api.sla2_packed_workspace_bytes(p, True) <= n + (1 << 30) + 2048
    p = api.make_packed_params(1, 1 << 25, 128, 1, 1, 64)                     # one tile of keys: 128 parts of it
    assert api.sla2_packed_workspace_bytes(p, True) > 2 * 128 * 128 * 64 * 4


def test_bad_packed_pointers():
    p = packed()
    for name in ("q", "k", "v", "q_start", "k_start", "out"):
        assert forward(p, **{name: None}) == EINVAL, name
    for name in ("q", "k", "v", "q_start", "k_start", "out", "lse", "dout", "dq", "dk", "dv"):
        assert backward(p, **{name: None}) == EINVAL, name
    for kw in (dict(q=Q + 8), dict(k=K + 2), dict(v=V + 4), dict(out=OUT + 8), dict(q_start=QS + 2), dict(k_start=KS + 1), dict(lse=LSE + 2)):
        assert forward(p, **kw) == EINVAL and backward(p, **kw) == EINVAL, kw
    for kw in (dict(dout=DO + 8), dict(dq=DQ + 2), dict(dk=DK + 8), dict(dv=DV + 4)):
        assert backward(p, **kw) == EINVAL, kw
    assert api._lib.sla2_packed_workspace_bytes(ctypes.byref(p), 2) == 0
    for fn, need in ((forward, api.sla2_packed_workspace_bytes(p)), (backward, api.sla2_packed_workspace_bytes(p, True))):
        assert need > 0
        for kw in (dict(workspace=None), dict(workspace=WS + 16), dict(ws_bytes=need - 1), dict(ws_bytes=0)):
            assert fn(p, **kw) == EWORKSPACE, kw


def test_packed_aliases():
    p, size, kv = packed(), 10 * 4 * 64 * 2, 12 * 2 * 64 * 2
    for kw in (dict(out=Q), dict(out=K), dict(out=V + kv - 16), dict(out=Q + size - 16), dict(out=QS), dict(lse=Q), dict(lse=OUT),
               dict(lse=KS), dict(workspace=Q), dict(workspace=OUT), dict(workspace=LSE)):
        assert forward(p, **kw) == EALIAS, kw
    for kw in (dict(dq=Q), dict(dq=DO), dict(dk=K), dict(dk=V), dict(dv=DK), dict(dv=DK + kv - 16), dict(dk=DQ), dict(dq=OUT), dict(dv=LSE),
               dict(dk=QS), dict(workspace=DQ), dict(workspace=LSE), dict(workspace=DO), dict(workspace=DV)):
        assert backward(p, **kw) == EALIAS, kw
    # slices of rows that hold q, k and v heads: apart, until one of them is moved by a head
    row = 8 * 64
    p = packed(tokens_k=10, q_stride=(64, row), kv_stride=(64, row))
    apart = dict(dq=DQ, dk=DQ + 4 * 64 * 2, dv=DQ + 6 * 64 * 2, ws_bytes=0)
    assert backward(p, **apart) == EWORKSPACE
    assert backward(p, **dict(apart, dk=DQ + 3 * 64 * 2)) == EALIAS
    assert backward(p, **dict(apart, dv=DQ + 7 * 64 * 2)) == EALIAS
    assert backward(p, **dict(apart, q=DQ + 5 * 64 * 2)) == EALIAS


def test_packed_tensors_that_are_refused():
    """What the binding sees of tensors: another type, too few elements, not contiguous, on the host."""
    t = torch.zeros(10, 4, 64, dtype=torch.bfloat16)
    assert forward(packed(), q=t) == EINVAL                        # on the host
    for bad in (t.float(), t[:9], torch.zeros(4, 10, 64, dtype=torch.bfloat16).transpose(0, 1)):
        assert forward(packed(), q=bad) == EINVAL
    assert forward(packed(), q_start=torch.zeros(4, dtype=torch.int64)) == EINVAL


def test_dout_in_an_order_of_its_own():
    """out head-major, dout token-major: each is held to its own strides, in what is refused and in what may overlap."""
    for kw, status in ((dict(dout_stride=(64, 0)), EINVAL), (dict(dout_stride=(0, 256)), EINVAL), (dict(dout_stride=(-64, 256)), EINVAL),
                       (dict(dout_stride=(68, 256)), EUNSUPPORTED), (dict(dout_stride=(64, 56)), EUNSUPPORTED),
                       (dict(dout_stride=(64, 1 << 24)), EUNSUPPORTED)):
        p = packed(**kw)
        assert api.sla2_packed_workspace_bytes(p, True) == 0 and backward(p) == status, kw
    size = 10 * 4 * 64 * 2
    p = packed(out_stride=(10 * 64, 64), dout_stride=(128, 512))             # dout: 9 x 512 + 3 x 128 + 64 elements, 10,112 bytes
    assert backward(p, ws_bytes=0) == EWORKSPACE
    assert backward(p, dq=DO + size, ws_bytes=0) == EALIAS                     # past what it would have with the strides of out
    assert backward(p, dq=OUT + size, ws_bytes=0) == EWORKSPACE
    assert backward(packed(out_stride=(128, 512)), dq=DO + size, ws_bytes=0) == EALIAS        # not stated: those of out


def test_strides_that_a_view_brings():
    """The backward call of the binding states the strides of out and dout where they are views in another order; not those of a value or a row
    that stands for all, which stay refused."""
    T, H, d = 10, 4, 64
    plain, heads = torch.zeros(T, H, d, dtype=torch.bfloat16), torch.zeros(H, T, d, dtype=torch.bfloat16).transpose(0, 1)
    rows = torch.zeros(T, 3, H, d, dtype=torch.bfloat16)[:, 1]

    def stated(out, dout):
        p = api._with_strides_of(packed(), out, dout)
        return tuple(p.out_stride), tuple(p.dout_stride)
    flat = (d, H * d)
    assert stated(heads, plain) == ((T * d, d), flat) and stated(plain, heads) == (flat, (T * d, d)) and stated(rows, heads) == ((d, 3 * H * d), (T * d, d))
    assert stated(OUT, heads) == (flat, (T * d, d))                            # an address is taken as it is: contiguous
    nothing = ((0, 0), (0, 0))
    for bad in (torch.zeros((), dtype=torch.bfloat16).expand(T, H, d), torch.zeros(d, dtype=torch.bfloat16).expand(T, H, d),
                torch.zeros(T, 1, d, dtype=torch.bfloat16).expand(T, H, d), torch.zeros(T, H, 2 * d, dtype=torch.bfloat16)[..., ::2],
                torch.zeros(T + 1, H, 2 * d, dtype=torch.bfloat16)[..., :d], torch.zeros(T, 2 * H * d, dtype=torch.bfloat16)[:, ::2]):
        assert stated(plain, bad) == nothing and stated(bad, plain) == nothing
    assert not api._is_view(plain) and not api._is_view(OUT) and not api._is_view(None) and api._is_view(heads)


# ---- cache ----
KC, VC, SK, SV, FIRST, TABLE, LEN = (i << 28 for i in range(1, 8))
FP8, INT8, NONE = api.SLA2_QUANT_FP8, api.SLA2_QUANT_INT8, api.SLA2_QUANT_NONE


def cache(**kw):
    return api.make_cache_params(**dict(dict(B=3, H=4, H_kv=2, d=64, pages=10, page_size=16, max_pages=4, tokens=7, quant_mode=FP8), **kw))


def write(p, **kw):
    a = dict(dict(k=K, v=V, page_table=TABLE, k_cache=KC, v_cache=VC, k_scale=SK, v_scale=SV, start=QS, first=FIRST), **kw)
    return api.sla2_cache_write(p, check=False, **a)


def read(p, **kw):
    a = dict(dict(k=K, v=V, page_table=TABLE, k_cache=KC, v_cache=VC, k_scale=SK, v_scale=SV, start=QS, first=FIRST), **kw)
    return api.sla2_cache_read(p, check=False, **a)


def attention(p, **kw):
    a = dict(dict(q=Q, k_cache=KC, v_cache=VC, page_table=TABLE, length=LEN, out=OUT, k_scale=SK, v_scale=SV, lse=LSE, workspace=WS, ws_bytes=BIG), **kw)
    return api.sla2_cache_attention(p, check=False, **a)


@pytest.mark.parametrize("kw,status", [
    (dict(B=0), EINVAL), (dict(pages=0), EINVAL), (dict(max_pages=0), EINVAL), (dict(tokens=-1), EINVAL), (dict(H=0), EINVAL),
    (dict(H=5), EINVAL), (dict(H_kv=0), EINVAL), (dict(d=32), EUNSUPPORTED), (dict(dtype=0), EUNSUPPORTED), (dict(dtype=7), EINVAL),
    (dict(page_size=0), EUNSUPPORTED), (dict(page_size=8), EUNSUPPORTED), (dict(page_size=48), EUNSUPPORTED), (dict(page_size=512), EUNSUPPORTED),
    (dict(page_size=-16), EUNSUPPORTED), (dict(quant_mode=4), EINVAL), (dict(quant_mode=-1), EINVAL),
    (dict(quant_mode=api.SLA2_QUANT_FP8_V), EUNSUPPORTED), (dict(scale=-0.5), EINVAL), (dict(scale=float("nan")), EINVAL),
    (dict(B=65536), EUNSUPPORTED), (dict(max_pages=1 << 27), EUNSUPPORTED), (dict(table_stride=3), EINVAL), (dict(table_stride=-4), EINVAL),
    (dict(cache_stride=(2048, 1024, 0)), EINVAL), (dict(cache_stride=(2048, 1024, 48)), EUNSUPPORTED), (dict(cache_stride=(2056, 1024, 64)), EUNSUPPORTED),
    (dict(cache_stride=(1 << 40, 1024, 64)), EUNSUPPORTED), (dict(cache_stride=(2048, 1024, 1 << 24)), EUNSUPPORTED),
    (dict(kv_stride=(64, 0)), EINVAL), (dict(q_stride=(60, 256)), EUNSUPPORTED), (dict(out_stride=(64, 32)), EUNSUPPORTED),
    (dict(tokens=1 << 30), EUNSUPPORTED),
])
def test_bad_cache_parameters(kw, status):
    p = cache(**kw)
    assert api.sla2_cache_workspace_bytes(p) == 0
    assert write(p) == status and read(p) == status and attention(p) == status


def test_most_rows_of_a_call():
    """64 rows a workgroup of 256 threads: below 2^32 threads, what a launch may have."""
    assert api.sla2_cache_workspace_bytes(cache(tokens=(1 << 30) - 64)) > 0
    p = cache(tokens=(1 << 30) - 63)
    assert api.sla2_cache_workspace_bytes(p) == 0 and write(p) == EUNSUPPORTED and read(p) == EUNSUPPORTED


def test_bad_cache_pointers():
    p = cache()
    for fn, names in ((write, ("k", "v")), (read, ("k", "v")), (attention, ("q", "out", "length"))):
        for name in names + ("page_table", "k_cache", "v_cache", "k_scale", "v_scale"):
            assert fn(p, **{name: None}) == EINVAL, (fn, name)
        for kw in (dict(k_cache=KC + 8), dict(v_cache=VC + 1), dict(k_scale=SK + 8), dict(v_scale=SV + 4), dict(page_table=TABLE + 2)):
            assert fn(p, **kw) == EINVAL, (fn, kw)
    for fn in (write, read):
        for kw in (dict(k=K + 8), dict(v=V + 2), dict(start=QS + 2), dict(first=FIRST + 3), dict(start=None)):   # the last: 7 rows for 3 sequences
            assert fn(p, **kw) == EINVAL, kw
    for kw in (dict(q=Q + 8), dict(out=OUT + 2), dict(length=LEN + 1), dict(lse=LSE + 2)):
        assert attention(p, **kw) == EINVAL, kw
    plain = cache(quant_mode=NONE)
    assert write(plain) == EINVAL and read(plain, k_scale=None) == EINVAL and attention(plain, v_scale=None) == EINVAL   # scales without codes
    need = api.sla2_cache_workspace_bytes(p)
    assert need > 0
    for kw in (dict(workspace=None), dict(workspace=WS + 16), dict(ws_bytes=need - 1)):
        assert attention(p, **kw) == EWORKSPACE, kw


def test_cache_aliases():
    p = cache()
    size, scales, rows = 10 * 2 * 16 * 64, 10 * 2 * 16 * 4, 7 * 2 * 64 * 2
    for kw in (dict(k_cache=K), dict(v_cache=V), dict(v_cache=KC), dict(v_cache=KC + size - 16), dict(k_scale=KC), dict(v_scale=SK),
               dict(v_scale=SK + scales - 16), dict(k_scale=QS), dict(v_scale=FIRST), dict(k_cache=TABLE)):
        assert write(p, **kw) == EALIAS, kw
    for kw in (dict(k=KC), dict(v=VC), dict(v=K), dict(v=K + rows - 16), dict(k=SK), dict(k=QS), dict(v=FIRST), dict(k=TABLE)):
        assert read(p, **kw) == EALIAS, kw
    for kw in (dict(out=KC), dict(out=VC + size - 16), dict(out=SK), dict(out=LEN), dict(out=TABLE), dict(lse=Q), dict(lse=OUT), dict(workspace=Q),
               dict(workspace=OUT), dict(workspace=SV), dict(workspace=LSE), dict(out=Q + 16)):
        assert attention(p, **kw) == EALIAS, kw
    # keys and values as the two halves of every page
    both = cache(cache_stride=(2 * 2 * 16 * 64, 16 * 64, 64))
    assert attention(both, k_cache=KC, v_cache=KC + 2 * 16 * 64, ws_bytes=0) == EWORKSPACE
    assert write(both, k_cache=KC, v_cache=KC + 16 * 64) == EALIAS


def test_cache_tensors_that_are_refused():
    p = cache()
    for bad in (torch.zeros(10, 2, 16, 64, dtype=torch.int8), torch.zeros(9, 2, 16, 64, dtype=torch.uint8), torch.zeros(10, 2, 16, 64)):
        assert attention(p, k_cache=bad) == EINVAL
    assert write(p, page_table=torch.zeros(3, 4, dtype=torch.int64)) == EINVAL
    assert write(p, page_table=torch.zeros(2, 4, dtype=torch.int32)) == EINVAL


def test_a_page_table_of_stated_stride_has_its_elements(monkeypatch):
    """A table with room between its rows is held to its B max_pages elements, as other strided tensors are to theirs."""
    seen = []
    monkeypatch.setattr(api, "_call", lambda fn, params, tensors, *rest: seen.append(tensors) or 0)
    p, t = cache(table_stride=9), torch.zeros(3, 9, dtype=torch.int32)[:, :4]
    for fn in (write, read, attention):
        assert fn(p, page_table=t) == 0
        (_, dtype, count, dense), = [x for x in seen.pop() if x[0] is t]
        assert (dtype, count, dense) == (torch.int32, 12, False) and t.numel() == count
