"""sla2_packed_forward and sla2_packed_backward against the fp64 oracle, element by element, with the bounds of stream_helpers."""
import numpy as np
import pytest

import stream_oracle as S
from stream_helpers import HALF, UNIT, close, dev, f64, guards_ok, lse_bound, out_bound, rows_like, starts, tiny, weight_error

pytestmark = pytest.mark.gpu


def run(lens_q, lens_k, H, Hkv, d, causal, layout="plain", scale=0.0, seed=0, lead=0, behind=0, edit=None, by=1.0, backward=True):
    """A forward and a backward call, checked.  lead, behind: rows in front of the first and behind the last sequence."""
    import torch
    from paper_2602_12675_amd import api
    gen = torch.Generator(device="cuda").manual_seed(seed)
    Tq, Tk = lead + sum(lens_q) + behind, lead + sum(lens_k) + behind
    q, sq, _ = rows_like(Tq, H, d, layout, gen, by)
    k, sk, _ = rows_like(Tk, Hkv, d, layout, gen)
    v, _, _ = rows_like(Tk, Hkv, d, layout, gen)
    out, so, obuf = rows_like(Tq, H, d, layout)
    dout, _, _ = rows_like(Tq, H, d, layout, gen)
    lse = torch.full((H, Tq), 7.0, device="cuda")
    qs, ks = starts(lens_q, lead), starts(lens_k, lead)
    if edit:
        edit(q, k, v, dout, qs, ks)
    p = api.make_packed_params(len(lens_q), Tq, Tk, H, Hkv, d, causal=causal, scale=scale, q_stride=sq, kv_stride=sk, out_stride=so)
    tqs, tks = dev(qs), dev(ks)
    ws = torch.empty(api.sla2_packed_workspace_bytes(p, True), dtype=torch.uint8, device="cuda").fill_(255)
    api.sla2_packed_forward(p, q, k, v, tqs, tks, out, lse=lse, workspace=ws)
    torch.cuda.synchronize()
    real = scale or d ** -0.5
    ref = S.packed_forward(f64(q), f64(k), f64(v), qs, ks, causal, real)
    inside = ~np.isnan(ref["out"][:, 0, 0])
    n = max(lens_k) if lens_k else 0
    r = weight_error(d, n, ref["smag"])                            # [H, Tq]
    close(out[dev(inside, torch.bool)], ref["out"][inside], out_bound(ref["out"], ref["mag"], r.T[..., None])[inside], "out")
    close(lse[:, dev(inside, torch.bool)], ref["lse"][:, inside], lse_bound(ref["lse"], r)[:, inside], "lse")
    assert bool((out[dev(~inside, torch.bool)] == 7).all()) and bool((lse[:, dev(~inside, torch.bool)] == 7).all())
    guards_ok(layout, obuf, H, d)
    if not backward:
        return p, (q, k, v, tqs, tks, out, lse, dout), ref
    dq, _, qbuf = rows_like(Tq, H, d, layout)
    dk, _, kbuf = rows_like(Tk, Hkv, d, layout)
    dv, _, vbuf = rows_like(Tk, Hkv, d, layout)
    ws.fill_(255)
    api.sla2_packed_backward(p, q, k, v, tqs, tks, out, lse, dout, dq, dk, dv, workspace=ws)
    torch.cuda.synchronize()
    b = S.packed_backward(f64(q), f64(k), f64(v), qs, ks, causal, real, f64(out), f64(lse), f64(dout))
    rows = (H // Hkv) * max(lens_q + [0])
    e = weight_error(d, max(rows, n), b["smag"])
    for name, got, member in (("dq", dq, qs), ("dk", dk, ks), ("dv", dv, ks)):
        sel = slice(member[0], member[-1])
        small = b[name + "_small"][sel] if name != "dv" else 0.0
        bound = HALF * np.abs(b[name][sel]) + (1 + HALF) * ((HALF + e) * b[name + "_mag"][sel] + UNIT * (d + 8) * small) + tiny(max(rows, n), f64(k if name == "dq" else q if name == "dk" else dout))
        close(got[sel], b[name][sel], bound, name)
        assert bool((got[:member[0]] == 7).all()) and bool((got[member[-1]:] == 7).all()), name
    guards_ok(layout, qbuf, H, d)
    guards_ok(layout, kbuf, Hkv, d)
    guards_ok(layout, vbuf, Hkv, d)
    return p, (q, k, v, tqs, tks, out, lse, dout, dq, dk, dv), ref


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [1, 2, 31, 63, 64, 65, 127, 128, 129, 257, 300])
def test_lengths(n, d, causal):
    run([n], [n], 2, 1, d, causal, seed=n)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens", [([5, 1, 200, 33], [5, 1, 200, 33]), ([1, 3, 40], [300, 64, 129]), ([130, 70, 5], [3, 1, 64]),
                                  ([7, 0, 9], [7, 12, 0]), ([0, 0, 3], [0, 4, 3]), ([64, 129], [0, 0])])
def test_packed_sequences(lens, d, causal):
    run(*lens, 3, 3, d, causal)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("heads", [(8, 1), (6, 2), (5, 5), (20, 1)])
@pytest.mark.parametrize("layout", ["plain", "padded", "heads"])
def test_groups_and_layouts(heads, layout, causal):
    run([70, 2, 131], [90, 2, 131], *heads, 64 if heads[0] > 8 else 128, causal, layout, seed=4)


def test_rows_outside_of_sequences_are_left():
    run([9, 130], [70, 3], 2, 2, 128, False, lead=3, behind=5)
    run([9, 130], [9, 130], 2, 1, 64, True, lead=130, behind=200)


def test_many_short_sequences():
    lens = [(7 * i) % 5 for i in range(150)]
    run(lens, lens, 2, 1, 64, True)
    run(lens, [(3 * i) % 4 for i in range(150)], 1, 1, 128, False)


def test_scale_and_large_scores():
    run([65], [130], 2, 2, 64, False, scale=0.7)
    run([65], [130], 2, 1, 128, True, scale=1.5, by=4.0)           # rows of one weight; references that move by thousands


def test_keys_rise_along_the_sequence():
    """The running maximum moves at every step."""
    def edit(q, k, v, dout, qs, ks):
        import torch
        q.fill_(1.0)
        k.copy_((torch.arange(k.shape[0], device="cuda")[:, None, None] * 0.05).expand_as(k))
    run([33], [400], 1, 1, 64, False, edit=edit)
    run([400], [400], 1, 1, 128, True, edit=edit)


def test_what_is_not_finite_stays_in_its_sequence():
    def edit(q, k, v, dout, qs, ks):
        k[ks[1]:ks[2], 0, 3] = float("nan")
        v[ks[1]:ks[2], 0, 5] = float("inf")
        q[qs[1]:qs[2]] = float("nan")
        dout[qs[1]:qs[2]] = float("nan")
    import torch
    from paper_2602_12675_amd import api
    for lens, causal in (([40, 30, 50], False), ([64, 64, 64], True), ([1, 1, 1], False)):
        clean = run(lens, lens, 2, 1, 64, causal, seed=9)[1]
        with_nan = [t.clone() for t in clean[:3]] + [clean[7].clone()]
        q, k, v, dout = with_nan
        qs = starts(lens)
        edit(q, k, v, dout, qs, qs)
        p = api.make_packed_params(3, sum(lens), sum(lens), 2, 1, 64, causal=causal)
        ws = torch.empty(api.sla2_packed_workspace_bytes(p, True), dtype=torch.uint8, device="cuda")
        out, lse = torch.zeros_like(clean[5]), torch.zeros_like(clean[6])
        api.sla2_packed_forward(p, q, k, v, clean[3], clean[4], out, lse=lse, workspace=ws)
        keep = torch.ones(sum(lens), dtype=torch.bool, device="cuda")
        keep[qs[1]:qs[2]] = False
        assert torch.equal(out[keep], clean[5][keep]) and torch.equal(lse[:, keep], clean[6][:, keep])
        assert bool(torch.isnan(out[~keep]).any())
        dq, dk, dv = (torch.zeros_like(t) for t in clean[8:11])
        api.sla2_packed_backward(p, q, k, v, clean[3], clean[4], out, lse, dout, dq, dk, dv, workspace=ws)
        for got, want in zip((dq, dk, dv), clean[8:11]):
            assert torch.equal(got[keep], want[keep]) and bool(torch.isnan(got[~keep]).any())


def test_offsets_that_do_not_fit_stay_inside():
    """Descending, negative and too large offsets: each sequence is what is left of it inside the tensors."""
    import torch
    from paper_2602_12675_amd import api
    q, k, v = (torch.randn(100, 1, 64, device="cuda").bfloat16() for _ in range(3))
    buf = torch.full((140, 1, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    out = buf[20:120]
    p = api.make_packed_params(3, 100, 100, 1, 1, 64)
    ws = torch.empty(api.sla2_packed_workspace_bytes(p, True), dtype=torch.uint8, device="cuda")
    lse = torch.zeros(1, 100, device="cuda")
    for qs in ([-5, 20, 10, 400], [90, 50, 2 ** 31 - 1, -2 ** 31], [0, 200, 300, 400]):
        api.sla2_packed_forward(p, q, k, v, dev(qs), dev(qs), out, lse=lse, workspace=ws)
        dq, dk, dv = (torch.zeros_like(q) for _ in range(3))
        api.sla2_packed_backward(p, q, k, v, dev(qs), dev(qs), out, lse, q, dq, dk, dv, workspace=ws)
        torch.cuda.synchronize()
        assert bool((buf[:20] == 7).all()) and bool((buf[120:] == 7).all())


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("size", [(100, 100, 2, 1), (1500, 1100, 8, 1), (41, 2604, 4, 1), (1503, 1503, 3, 3), (4303, 209, 16, 1)])
def test_offsets_that_do_not_fit_write_nothing_else(size, causal, d):
    """Sequences that overlap, descend, begin below 0 or end behind the tensors, grouped heads, rows and keys dealt to several workgroups and
    launches of both kinds: nothing around out, lse, the gradients and the workspace changes."""
    import torch
    from paper_2602_12675_amd import api
    Tq, Tk, H, Hkv = size
    gen = torch.Generator(device="cuda").manual_seed(1)
    q, g = (torch.randn((Tq, H, d), generator=gen, device="cuda").bfloat16() for _ in range(2))
    k, v = (torch.randn((Tk, Hkv, d), generator=gen, device="cuda").bfloat16() for _ in range(2))
    p = api.make_packed_params(4, Tq, Tk, H, Hkv, d, causal=causal)
    room = 1 << 13
    guarded = []

    def inside(shape, dtype, fill):
        n = int(np.prod(shape))
        buf = torch.full((n + 2 * room,), fill, dtype=dtype, device="cuda")
        guarded.append((buf, n, fill))
        return buf[room:room + n].view(shape)
    out, dq = (inside((Tq, H, d), torch.bfloat16, 7.0) for _ in range(2))
    dk, dv = (inside((Tk, Hkv, d), torch.bfloat16, 7.0) for _ in range(2))
    lse = inside((H, Tq), torch.float32, 7.0)
    ws = [inside((api.sla2_packed_workspace_bytes(p, x),), torch.uint8, 0x77) for x in (False, True)]

    def offsets(T):
        far = 2 ** 31 - 1
        return [[0, T // 3, T // 4, T + 50, T], [-7, T, 0, T, far], [T // 2, T // 4, far, -far - 1, T // 8], [0, T, 0, T, 0],
                [0, 1, T - 1, T, T], [far, -1, far, -1, far], [T, T // 2, T // 3, T // 4, 0]]
    for qs, ks in [(a, b) for i, a in enumerate(offsets(Tq)) for j, b in enumerate(offsets(Tk)) if (i + j) % 3 == 0 or i == j]:
        tqs, tks = dev(qs), dev(ks)
        api.sla2_packed_forward(p, q, k, v, tqs, tks, out, lse=lse, workspace=ws[0])
        api.sla2_packed_backward(p, q, k, v, tqs, tks, out, lse, g, dq, dk, dv, workspace=ws[1])
        torch.cuda.synchronize()
        for buf, n, fill in guarded:
            assert bool((buf[:room] == fill).all()) and bool((buf[room + n:] == fill).all()), (qs, ks)


def test_gradients_in_one_buffer_and_empty_sides():
    """dq, dk and dv as slices of the gradient of one projection, with other numbers of heads; no queries, no keys."""
    import torch
    from paper_2602_12675_amd import api
    T, H, Hkv, d = 77, 6, 2, 64
    p, t, _ = run([T], [T], H, Hkv, d, True)
    q, k, v, qs, ks, out, lse, dout, dq, dk, dv = t
    row = (H + 2 * Hkv) * d
    buf = torch.zeros((T, H + 2 * Hkv, d), dtype=torch.bfloat16, device="cuda")
    qkv = torch.cat([q, k, v], 1)
    p2 = api.make_packed_params(1, T, T, H, Hkv, d, causal=True, q_stride=(d, row), kv_stride=(d, row))
    ws = torch.empty(api.sla2_packed_workspace_bytes(p2, True), dtype=torch.uint8, device="cuda")
    api.sla2_packed_backward(p2, qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:], qs, ks, out, lse, dout, buf[:, :H], buf[:, H:H + Hkv],
                             buf[:, H + Hkv:], workspace=ws)
    assert torch.equal(buf, torch.cat([dq, dk, dv], 1))
    none, zero = torch.empty((0, H, d), dtype=torch.bfloat16, device="cuda"), dev([0, 0])
    p3 = api.make_packed_params(1, 0, T, H, Hkv, d)
    e = torch.empty((H, 0), device="cuda")
    dk.fill_(1), dv.fill_(1)
    api.sla2_packed_forward(p3, None, k, v, zero, ks, None, workspace=ws)
    api.sla2_packed_backward(p3, None, k, v, zero, ks, None, None, None, None, dk, dv, workspace=ws)
    assert not bool(dk.any()) and not bool(dv.any()) and none.numel() == e.numel() == 0
    p4 = api.make_packed_params(1, T, 0, H, Hkv, d)
    ws = torch.empty(api.sla2_packed_workspace_bytes(p4, True), dtype=torch.uint8, device="cuda")
    api.sla2_packed_forward(p4, q, None, None, qs, zero, out, lse=lse, workspace=ws)
    assert not bool(out.any()) and bool((lse == -float("inf")).all())
    api.sla2_packed_backward(p4, q, None, None, qs, zero, out, lse, dout, dq, None, None, workspace=ws)
    assert not bool(dq.any())


@pytest.mark.parametrize("case", [([70, 2, 131], [90, 2, 131], 6, 2, 64, True), ([300, 41], [1500, 900], 2, 2, 128, False), ([40, 1], [2600, 4], 4, 1, 64, True),
                                  ([4300, 3], [200, 9], 16, 1, 128, False), ([2300], [150], 32, 32, 64, False)])
def test_out_and_dout_in_orders_of_their_own(case):
    """What the forward pass kept is head-major, what the loss hands back token-major, or the other way around: the same bits as of contiguous
    copies, by strides that are stated and by those of the views.  All launches of the backward pass are reached."""
    import torch
    from paper_2602_12675_amd import api
    p, t, _ = run(*case)
    q, k, v, qs, ks, out, lse, dout, dq, dk, dv = t
    T, H, d = q.shape
    ws = torch.empty(api.sla2_packed_workspace_bytes(p, True), dtype=torch.uint8, device="cuda")

    def of(layout, x):
        y, st, _ = rows_like(T, H, d, layout)
        y.copy_(x)
        return y, st or (d, H * d)
    for a, b in (("heads", "plain"), ("plain", "heads"), ("padded", "heads"), ("heads", "padded")):
        (o, so), (g, sg) = of(a, out), of(b, dout)
        stated = api.make_packed_params(p.sequences, T, k.shape[0], H, k.shape[1], d, causal=bool(p.causal), out_stride=so, dout_stride=sg)
        for params in (p, stated):
            got = [torch.full_like(x, 5) for x in (dq, dk, dv)]
            ws.fill_(255)
            api.sla2_packed_backward(params, q, k, v, qs, ks, o, lse, g, *got, workspace=ws)
            for x, y in zip(got, (dq, dk, dv)):
                assert torch.equal(x, y), (a, b)
    one = torch.ones((), dtype=torch.bfloat16, device="cuda").expand(T, H, d)
    assert api.sla2_packed_backward(p, q, k, v, qs, ks, out, lse, one, dq, dk, dv, workspace=ws, check=False) == api.SLA2_EINVAL


@pytest.mark.parametrize("case", [([700], [700], 4, 2, 128, True), ([300, 41], [1500, 900], 2, 2, 64, False), ([9], [5000], 2, 1, 128, False),
                                  ([1], [3000], 4, 4, 64, True), ([2500], [70], 3, 3, 128, False), ([1200], [1200], 2, 1, 64, True),
                                  ([5, 900, 1], [5, 2000, 700], 8, 2, 128, True)])
def test_longer_sequences_and_the_same_bits_twice(case):
    import torch
    from paper_2602_12675_amd import api
    p, t, _ = run(*case)
    q, k, v, qs, ks, out, lse, dout, dq, dk, dv = t
    again = [torch.zeros_like(x) for x in (out, lse, dq, dk, dv)]
    ws = torch.empty(api.sla2_packed_workspace_bytes(p, True), dtype=torch.uint8, device="cuda")
    api.sla2_packed_forward(p, q, k, v, qs, ks, again[0], lse=again[1], workspace=ws)
    api.sla2_packed_backward(p, q, k, v, qs, ks, out, lse, dout, *again[2:], workspace=ws)
    for x, y in zip(again, (out, lse, dq, dk, dv)):
        assert torch.equal(x, y)


@pytest.mark.parametrize("seed", range(16))
def test_random_shapes(seed):
    """A sample of the parameter space: lengths around the tiles, groups, strides, masks, both head dimensions."""
    rng = np.random.default_rng(1000 + seed)
    S = int(rng.choice([1, 2, 3, 7]))
    Hkv, group = [(1, 1), (2, 3), (1, 8), (3, 2), (2, 16), (1, 5)][int(rng.integers(6))]
    edge = [0, 1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 200, 320, 513]
    lens_k = [int(rng.choice(edge)) for _ in range(S)]
    lens_q = [int(rng.choice(edge[:12])) for _ in range(S)] if rng.random() < 0.6 else list(lens_k)
    lens_q[0], lens_k[0] = max(1, lens_q[0]), max(1, lens_k[0])
    run(lens_q, lens_k, Hkv * group, Hkv, int(rng.choice([64, 128])), bool(rng.integers(2)), str(rng.choice(["plain", "padded", "heads"])), seed=seed,
        lead=int(rng.integers(3)), behind=int(rng.integers(4)))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_rows_that_fill_the_gpu(d, causal):
    """More tiles of rows than are at work at a time: rows and keys in launches of their own, keys whole, in parts, and of short sequences."""
    run([1 + i % 2 for i in range(40)], [1 + i % 3 for i in range(40)], 16, 16, d, causal)
    run([4300, 3], [200, 9], 16, 1, d, causal, layout="heads" if causal else "padded")
    run([(5 * i) % 7 for i in range(300)], [(3 * i) % 5 for i in range(300)], 4, 2, d, causal)


@pytest.mark.parametrize("d", [64, 128])
def test_rows_dealt_to_several_workgroups_with_a_mask(d):
    """Long rows over few tiles of keys and few rows over many keys: parts of both, some of them empty, and sequences without parts."""
    run([1500, 3, 0], [200, 900, 5], 8, 1, d, True)
    run([40, 1], [2600, 4], 4, 1, d, True)
    run([1, 1, 700], [1, 2200, 0], 6, 2, d, False)


@pytest.mark.parametrize("d", [64, 128])
def test_scores_far_below_zero(d):
    """Scores around -1e34, powers of two all alike: no product rounds, and the result is the mean of the values."""
    def edit(q, k, v, dout, qs, ks):
        q.fill_(2.0 ** 59)
        k.fill_(-2.0 ** 50)
    p, (q, k, v, _, _, out, lse, _), ref = run([3, 70], [1, 200], 4, 2, d, False, edit=edit, backward=False)
    assert float(ref["lse"].max()) < -2e33
    mean = np.concatenate([np.repeat(f64(v[:1]), 3, 0), np.repeat(f64(v[1:]).mean(0, keepdims=True), 70, 0)]).repeat(2, 1)
    close(out, mean, HALF * np.abs(mean) + 300 * UNIT * float(v.float().abs().max()))   # P = 1 exactly; sums of 200 values in fp32
    close(lse, ref["lse"], 4 * UNIT * np.abs(ref["lse"]))


def test_offsets_past_32_bits():
    """5 GB of queries: rows at their end read the right keys and are written where they belong."""
    import torch
    from paper_2602_12675_amd import api
    T, H, d, n = 600_000, 32, 128, 70
    gen = torch.Generator(device="cuda").manual_seed(0)
    q = torch.zeros((T, H, d), dtype=torch.bfloat16, device="cuda")
    assert q.numel() > 2 ** 31
    q[-200:] = torch.randn((200, H, d), generator=gen, device="cuda").bfloat16()
    k, v = (torch.randn((2 * n, 4, d), generator=gen, device="cuda").bfloat16() for _ in range(2))
    out = torch.full_like(q, 7.0)
    p = api.make_packed_params(2, T, 2 * n, H, 4, d)
    ws = torch.empty(api.sla2_packed_workspace_bytes(p), dtype=torch.uint8, device="cuda")
    api.sla2_packed_forward(p, q, k, v, dev([0, T - 100, T]), dev([0, n, 2 * n]), out, workspace=ws)
    r = S.packed_forward(f64(q[-200:]), f64(k), f64(v), [0, 100, 200], [0, n, 2 * n], False, d ** -0.5)
    e = weight_error(d, n, r["smag"])
    close(out[-200:], r["out"], out_bound(r["out"], r["mag"], e.T[..., None]))
    close(out[:1].float(), np.repeat(f64(v[:n]).mean(0), 8, 0)[None], np.full((1, H, d), 2.0 ** -6))     # equal scores: the mean
