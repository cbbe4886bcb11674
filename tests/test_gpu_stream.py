"""Packed attention and the cache as a program uses them together: a stream whose frames are rotated, written into the cache, read by new
tokens and by later frames; calls on other streams; calls captured into graphs whose device arrays change between the replays."""
import numpy as np
import pytest

import layer_oracle as L
import stream_oracle as S
from paper_2602_12675_amd import workloads as W
from stream_helpers import HALF, UNIT, close, dev, f64, lse_bound, out_bound, weight_error

pytestmark = pytest.mark.gpu
QUANTS = ["none", "fp8", "int8"]


def codes(api, quant):
    return {"none": api.SLA2_QUANT_NONE, "fp8": api.SLA2_QUANT_FP8, "int8": api.SLA2_QUANT_INT8}[quant]


def new_cache(torch, pages, Hkv, page, d, quant):
    t = {"none": torch.bfloat16, "fp8": torch.float8_e4m3fn, "int8": torch.int8}[quant]
    kv = [torch.zeros((pages, Hkv, page, d), device="cuda").to(t) for _ in range(2)]
    return kv, [None, None] if quant == "none" else [torch.zeros((pages, Hkv, page), device="cuda") for _ in range(2)]


def stored(x, quant):
    """What the cache holds of rows x (fp64, exactly bf16 values) [.., d], and what reading them back gives"""
    if quant == "none":
        return x, x
    c, s = S.code_rows(x.astype(np.float32), quant)
    back = W.bf16_bits_to_f32(W.f32_to_bf16_bits(c * s[..., None])).astype(np.float64)
    return c.astype(np.float64) * s[..., None].astype(np.float64), back


@pytest.mark.parametrize("quant", QUANTS)
def test_frames_of_a_stream(quant):
    """Two streams of frames of 6 x 7 tokens.  Every frame: q and k of the packed projection rotated in place at the frame's own time
    (sla2_rope_forward with origin), k and v into the cache, then read back with all frames before, and the frame's queries attend to
    them (sla2_packed_forward).  At the end one new token of each stream attends to its cache (sla2_cache_attention)."""
    import torch
    from paper_2602_12675_amd import api
    B, H, d, Y, X, frames, page = 2, 4, 64, 6, 7, 3, 16
    n = Y * X
    gen = torch.Generator(device="cuda").manual_seed(3)
    need = -(-(frames * n + 1) // page)
    table = dev(np.random.default_rng(0).permutation(2 * need + 1)[:2 * need].reshape(2, need).tolist())
    kv, scale = new_cache(torch, 2 * need + 1, H, page, d, quant)
    held = [[np.zeros((0, H, d)), np.zeros((0, H, d))] for _ in range(B)]            # k, v as the cache has them
    back = [[np.zeros((0, H, d)), np.zeros((0, H, d))] for _ in range(B)]            # as they are read back
    axes = (10, 11, 11)

    def write(k, v, first, start):
        p = api.make_cache_params(B, H, H, d, 2 * need + 1, page, need, tokens=k.shape[0], quant_mode=codes(api, quant), kv_stride=(d, 3 * H * d))
        api.sla2_cache_write(p, k, v, table, *kv, k_scale=scale[0], v_scale=scale[1], start=start, first=dev([first] * B))
        torch.cuda.synchronize()
        kk, vv = f64(k).reshape(B, -1, H, d), f64(v).reshape(B, -1, H, d)
        for b in range(B):
            for x, t in enumerate((kk, vv)):
                h, r = stored(t[b], quant)
                held[b][x], back[b][x] = np.concatenate([held[b][x], h]), np.concatenate([back[b][x], r])

    for f in range(frames):
        qkv = torch.randn((B, n, 3, H, d), generator=gen, device="cuda").bfloat16()
        st = (n * 3 * H * d, d, 3 * H * d)                           # the projection's rows hold q, k and v
        r = api.make_rope_params(B, H, n, d, axes, grid=(1, Y, X), origin=(f, 0, 0), in_stride=st, out_stride=st)
        freq = api.sla2_rope_frequencies(r, 10000.0)
        q, k = qkv[:, :, 0].transpose(1, 2), qkv[:, :, 1].transpose(1, 2)
        plain = f64(q)
        api.sla2_rope_forward(r, q, k, freq.cuda(), q, k)
        turned, mag = L.rope_forward(plain, L.grid_positions(n, (1, Y, X), (f, 0, 0))[None], freq.numpy(), axes)
        close(q, turned, HALF * np.abs(turned) + 16 * UNIT * mag)   # cosine and sine, two products and a sum: 8 units each way at most
        write(qkv.view(B * n, 3, H, d)[:, 1], qkv.view(B * n, 3, H, d)[:, 2], f * n, dev([0, n, 2 * n]))
        m = (f + 1) * n                                              # tokens that each stream has by now
        p = api.make_cache_params(B, H, H, d, 2 * need + 1, page, need, tokens=B * m, quant_mode=codes(api, quant))
        ks, vs = (torch.zeros((B * m, H, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        api.sla2_cache_read(p, *kv, table, ks, vs, k_scale=scale[0], v_scale=scale[1], start=dev([0, m, 2 * m]))
        for x, t in enumerate((ks, vs)):
            np.testing.assert_array_equal(f64(t), np.concatenate([back[b][x] for b in range(B)]))
        a = api.make_packed_params(B, B * n, B * m, H, H, d, q_stride=(d, 3 * H * d))
        out = torch.zeros((B * n, H, d), dtype=torch.bfloat16, device="cuda")
        ws = torch.empty(api.sla2_packed_workspace_bytes(a), dtype=torch.uint8, device="cuda")
        qs = qkv.view(B * n, 3, H, d)[:, 0]
        api.sla2_packed_forward(a, qs, ks, vs, dev([0, n, 2 * n]), dev([0, m, 2 * m]), out, workspace=ws)
        ref = S.packed_forward(f64(qs), f64(ks), f64(vs), [0, n, 2 * n], [0, m, 2 * m], False, d ** -0.5)
        close(out, ref["out"], out_bound(ref["out"], ref["mag"], weight_error(d, m, ref["smag"]).T[..., None]))
    new = torch.randn((B, 3, H, d), generator=gen, device="cuda").bfloat16()
    write(new[:, 1], new[:, 2], frames * n, None)
    p = api.make_cache_params(B, H, H, d, 2 * need + 1, page, need, quant_mode=codes(api, quant), q_stride=(d, 3 * H * d))
    out = torch.zeros((B, H, d), dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(api.sla2_cache_workspace_bytes(p), dtype=torch.uint8, device="cuda")
    api.sla2_cache_attention(p, new[:, 0], *kv, table, dev([frames * n + 1] * B), out, k_scale=scale[0], v_scale=scale[1], workspace=ws)
    q = f64(new[:, 0])
    for b in range(B):
        for h in range(H):
            o, _, mag, sm = S.attend(q[b, h][None], held[b][0][:, h], held[b][1][:, h], np.ones((1, frames * n + 1), dtype=bool), d ** -0.5)
            close(out[b, h][None], o, out_bound(o, mag, weight_error(d, frames * n + 1, sm)[:, None]))


def test_new_token_as_a_packed_query():
    """The same token by both ways: over the cache, and as a packed query over what reading the cache gives (bf16: the same values)."""
    import torch
    from paper_2602_12675_amd import api
    B, H, Hkv, d, page, n = 3, 8, 2, 128, 64, [700, 1, 130]
    gen = torch.Generator(device="cuda").manual_seed(5)
    need = -(-max(n) // page)
    table = dev(np.arange(B * need).reshape(B, need).tolist())
    kv, _ = new_cache(torch, B * need, Hkv, page, d, "none")
    k, v = (torch.randn((sum(n), Hkv, d), generator=gen, device="cuda").bfloat16() for _ in range(2))
    start = dev([0, 700, 701, 831])
    p = api.make_cache_params(B, H, Hkv, d, B * need, page, need, tokens=sum(n))
    api.sla2_cache_write(p, k, v, table, *kv, start=start)
    q = torch.randn((B, H, d), generator=gen, device="cuda").bfloat16()
    got, other = torch.zeros_like(q), torch.zeros_like(q)
    lse, lse2 = torch.zeros((B, H), device="cuda"), torch.zeros((H, B), device="cuda")
    api.sla2_cache_attention(p, q, *kv, table, dev(n), got, lse=lse, workspace=torch.empty(api.sla2_cache_workspace_bytes(p), dtype=torch.uint8, device="cuda"))
    a = api.make_packed_params(B, B, sum(n), H, Hkv, d, causal=True)
    ws = torch.empty(api.sla2_packed_workspace_bytes(a), dtype=torch.uint8, device="cuda")
    api.sla2_packed_forward(a, q, k, v, dev([0, 1, 2, 3]), start, other, lse=lse2, workspace=ws)
    # both are within the same bound of the exact result: see stream_helpers, with the largest of the terms
    smag = float((q.float().abs().reshape(-1, d) @ k.float().abs().reshape(-1, d).T).max()) * d ** -0.5
    e, top = weight_error(d, max(n), smag), float(v.float().abs().max())
    assert float((got.float() - other.float()).abs().max()) <= 2 * (HALF + (HALF + e) * (1 + HALF)) * top
    assert float((lse - lse2.T).abs().max()) <= 2 * lse_bound(lse.cpu().numpy(), e).max()


def test_on_another_stream():
    """Inputs made on a side stream, calls put on it by the argument and as the current stream."""
    import torch
    from paper_2602_12675_amd import api
    T, H, d = 300, 4, 64
    side = torch.cuda.Stream()
    p = api.make_packed_params(1, T, T, H, H, d, causal=True)
    ws = torch.empty(api.sla2_packed_workspace_bytes(p, True), dtype=torch.uint8, device="cuda")
    base = [torch.randn((T, H, d), device="cuda").bfloat16() for _ in range(4)]
    st = dev([0, T])
    torch.cuda.synchronize()

    def both(x, stream):
        out, lse = torch.zeros_like(x[0]), torch.zeros((H, T), device="cuda")
        g = [torch.zeros_like(x[0]) for _ in range(3)]
        api.sla2_packed_forward(p, *x[:3], st, st, out, lse=lse, workspace=ws, stream=stream)
        api.sla2_packed_backward(p, *x[:3], st, st, out, lse, x[3], *g, workspace=ws, stream=stream)
        return [out, lse] + g

    want = both(base, None)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        late = []
        for t in base:
            u = torch.empty_like(t)
            torch.cuda._sleep(2_000_000)                           # the inputs arrive late on the side stream
            u.copy_(t)
            late.append(u)
        current = both(late, None)
        named = both(late, side)
    torch.cuda.synchronize()
    for a, b, c in zip(want, current, named):
        assert torch.equal(a, b) and torch.equal(a, c)


def test_packed_training_step_in_a_graph():
    """Forward and backward captured; offsets, inputs and workspace change between the replays, eager calls run in between."""
    import torch
    from paper_2602_12675_amd import api
    T, H, Hkv, d = 700, 6, 2, 128
    gen = torch.Generator(device="cuda").manual_seed(1)
    q, g = (torch.randn((T, H, d), generator=gen, device="cuda").bfloat16() for _ in range(2))
    k, v = (torch.randn((T, Hkv, d), generator=gen, device="cuda").bfloat16() for _ in range(2))
    p = api.make_packed_params(3, T, T, H, Hkv, d, causal=True)
    ws = torch.empty(api.sla2_packed_workspace_bytes(p, True), dtype=torch.uint8, device="cuda")
    start = dev([0, 300, 301, 700])
    bufs = [torch.zeros_like(q), torch.zeros((H, T), device="cuda"), torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)]

    def step(b, w):
        api.sla2_packed_forward(p, q, k, v, start, start, b[0], lse=b[1], workspace=w)
        api.sla2_packed_backward(p, q, k, v, start, start, b[0], b[1], g, *b[2:], workspace=w)

    step(bufs, ws)                                                  # warms up
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        step(bufs, ws)
    for rep, offsets in enumerate(([0, 300, 301, 700], [0, 0, 650, 700], [5, 100, 400, 600], [0, 300, 301, 700], [0, 700, 700, 700])):
        start.copy_(dev(offsets))
        q.add_(0.125 * rep)
        for b in bufs:
            b.fill_(3)
        ws.random_(0, 255)
        want = [torch.full_like(b, 3) for b in bufs]
        step(want, torch.empty_like(ws))                            # eager, with a workspace of its own
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(bufs, want):
            assert torch.equal(a, b), rep


@pytest.mark.parametrize("quant", QUANTS)
def test_decoding_steps_in_a_graph(quant):
    """A write and the attention captured once, replayed as the sequences grow; two graphs share a workspace."""
    import torch
    from paper_2602_12675_amd import api
    B, H, Hkv, d, page, cols = 5, 8, 2, 64, 16, 100
    gen = torch.Generator(device="cuda").manual_seed(2)
    table = dev(np.random.default_rng(1).permutation(B * cols).reshape(B, cols).tolist())
    kv, scale = new_cache(torch, B * cols, Hkv, page, d, quant)
    p = api.make_cache_params(B, H, Hkv, d, B * cols, page, cols, tokens=B, quant_mode=codes(api, quant))
    ws = torch.empty(api.sla2_cache_workspace_bytes(p), dtype=torch.uint8, device="cuda")
    q, out, out2 = (torch.zeros((B, H, d), dtype=torch.bfloat16, device="cuda") for _ in range(3))
    k, v = (torch.zeros((B, Hkv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    first, length = dev([0] * B), dev([1] * B)
    kw = dict(k_scale=scale[0], v_scale=scale[1])

    def write():
        api.sla2_cache_write(p, k, v, table, *kv, first=first, **kw)

    def attend(o, w):
        api.sla2_cache_attention(p, q, *kv, table, length, o, workspace=w, **kw)

    write(), attend(out, ws)
    torch.cuda.synchronize()
    side, graphs = torch.cuda.Stream(), [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    with torch.cuda.stream(side):
        with torch.cuda.graph(graphs[0], stream=side):
            write()
            attend(out, ws)
        with torch.cuda.graph(graphs[1], stream=side):
            attend(out2, ws)
    # sequences of other lengths from the beginning on, so that parts fall differently at each replay
    past = [0, 1500, 31, 1200, 700]
    n = sum(past)
    pk, pv = (torch.randn((n, Hkv, d), generator=gen, device="cuda").bfloat16() for _ in range(2))
    fill = api.make_cache_params(B, H, Hkv, d, B * cols, page, cols, tokens=n, quant_mode=codes(api, quant))
    api.sla2_cache_write(fill, pk, pv, table, *kv, start=dev([0] + np.cumsum(past).tolist()), **kw)
    for rep in range(5):
        at = [x + rep for x in past]
        first.copy_(dev(at)), length.copy_(dev([x + 1 for x in at]))
        for t in (q, k, v):
            t.copy_(torch.randn(t.shape, generator=gen, device="cuda"))
        ws.random_(0, 255)
        torch.cuda.synchronize()
        graphs[0].replay()
        graphs[1].replay()
        torch.cuda.synchronize()
        want = torch.zeros_like(out)
        attend(want, torch.empty_like(ws))
        assert torch.equal(out, want) and torch.equal(out2, want), rep
        write(), attend(want, ws)
        torch.cuda.synchronize()
        assert torch.equal(out, want), rep


@pytest.mark.parametrize("quant", QUANTS)
def test_a_stream_grows_in_a_table_reserved_for_it(quant):
    """One captured step, replayed from the first token on, in a table of 131,072 tokens; the workspace is never clean."""
    import torch
    from paper_2602_12675_amd import api
    B, H, Hkv, d, page, cols, own = 2, 8, 1, 128, 256, 512, 8                  # `own` pages of each sequence exist
    gen = torch.Generator(device="cuda").manual_seed(3)
    ids = np.full((B, cols), -1, dtype=np.int32)
    ids[:, :own] = np.random.default_rng(2).permutation(B * own).reshape(B, own)
    table = dev(ids.tolist())
    kv, scale = new_cache(torch, B * own, Hkv, page, d, quant)
    kw = dict(k_scale=scale[0], v_scale=scale[1])
    n = own * page
    k, v = (torch.randn((B * n, Hkv, d), generator=gen, device="cuda").bfloat16() for _ in range(2))
    fill = api.make_cache_params(B, H, Hkv, d, B * own, page, cols, tokens=B * n, quant_mode=codes(api, quant))
    api.sla2_cache_write(fill, k, v, table, *kv, start=dev([0, n, 2 * n]), **kw)
    p = api.make_cache_params(B, H, Hkv, d, B * own, page, cols, quant_mode=codes(api, quant))
    q = torch.randn((B, H, d), generator=gen, device="cuda").bfloat16()
    out, lse, length = torch.zeros_like(q), torch.zeros((B, H), device="cuda"), dev([1, 1])
    ws = torch.empty(api.sla2_cache_workspace_bytes(p), dtype=torch.uint8, device="cuda").fill_(255)

    def attend(o, w):
        api.sla2_cache_attention(p, q, *kv, table, length, o, lse=lse, workspace=w, **kw)

    attend(out, ws)
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        attend(out, ws)
    held = [[stored(f64(x[b * n:(b + 1) * n]), quant)[0] for x in (k, v)] for b in range(B)]
    for lengths in ([1, 1], [33, 2], [40, 100], [700, 33], [2000, 1500], [64, 2048], [2, 0]):
        length.copy_(dev(lengths))
        ws.fill_(255)
        out.fill_(3)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = torch.zeros_like(out)
        attend(want, torch.randint(0, 255, ws.shape, dtype=torch.uint8, device="cuda"))
        assert torch.equal(out, want), lengths
        for b, m in enumerate(lengths):
            for h in range(H):
                o, l_, mag, sm = S.attend(f64(q)[b, h][None], held[b][0][:m, 0], held[b][1][:m, 0], np.ones((1, m), dtype=bool), d ** -0.5)
                e = weight_error(d, max(m, 1), sm)
                close(out[b, h][None], o, out_bound(o, mag, e[:, None]))
                close(lse[b, h][None], l_, lse_bound(l_, e))
