"""Performance cases of attention over packed sequences of different lengths with grouped heads, forward and backward, and of a
paged cache of keys and values: writing it (with quantisation), reading it back, and the attention of one new token over it.

A case is a dict of plain values.  Lists of lengths are texts "a,b,c", one entry a sequence.
kind "packed" (forward) and "packed_bwd":
  H, H_kv, d      query head h reads key head h / (H / H_kv)
  q, k            lengths of the sequences in queries and in keys; tensors are [sum of lengths, heads, d], bf16
  causal          query i of n_q reads keys 0 .. i + n_k - n_q, otherwise all of its sequence
  joint           whether k and v are slices of one [tokens, 3, H_kv, d] projection
kind "write" and "read":
  H_kv, d, page   the cache is [pages, H_kv, page, d], pages of a sequence lie anywhere
  quant           "none" (bf16) | "fp8" (e4m3) | "int8", the latter two with a scale for each token and head
  lengths         tokens that a sequence has in the cache behind the call
  new             how many of them, the last ones, are written or read back
kind "decode":
  H, H_kv, d, page, quant, lengths     one new query of each sequence over its `lengths` tokens
"""
import math

import torch

own = False


def _packed(name, kind, H, H_kv, d, q, k, causal, joint):
    return {"name": name, "kind": kind, "H": H, "H_kv": H_kv, "d": d, "q": q, "k": k, "causal": causal, "joint": joint}


def _moved(name, kind, H_kv, d, page, quant, lengths, new):
    return {"name": name, "kind": kind, "H_kv": H_kv, "d": d, "page": page, "quant": quant, "lengths": lengths, "new": new}


def _decode(name, H, H_kv, d, page, quant, lengths):
    return {"name": name, "kind": "decode", "H": H, "H_kv": H_kv, "d": d, "page": page, "quant": quant, "lengths": lengths}


def _text(lengths):
    return ",".join(str(n) for n in lengths)


def _spread(n, lo, hi):
    """n lengths from lo to hi, evenly spread over their logarithm, long and short ones by turns."""
    all_ = [int(round(lo * (hi / lo) ** (i / (n - 1)))) for i in range(n)]
    return _text([all_[i * 37 % n] for i in range(n)] if n % 37 else all_)


def listed():
    return [
        # a batch of prompts in a text encoder of 16 heads: nothing but latency
        _packed("packed-prompts", "packed", 16, 16, 64, "77,5,31,1,64,12,49,18", "77,5,31,1,64,12,49,18", False, True),
        # video tokens of the smaller video model read the prompt, a guidance pair: a long prompt and a short one
        _packed("packed-prompt-to-video", "packed", 12, 12, 128, "32760,32760", "512,131", False, False),
        # stretches of a stream that see only what came before them, grouped heads, packed
        _packed("packed-causal-grouped", "packed", 40, 8, 128, "4096,2777,1021,1,297", "4096,2777,1021,1,297", True, False),
        # training: video tokens read the prompt
        _packed("packed-bwd-prompt-to-video", "packed_bwd", 12, 12, 128, "32760", "512", False, False),
        # training on packed stretches of a stream, grouped heads
        _packed("packed-bwd-causal-grouped", "packed_bwd", 40, 8, 128, "2048,4096,1021,1,1026", "2048,4096,1021,1,1026", True, False),
        # one new token of each of 64 sequences goes into the cache: latency
        _moved("write-tokens-int8", "write", 8, 128, 64, "int8", _spread(64, 17, 8192), _text([1] * 64)),
        # the keys and values of all latent frames of a 12-head model
        _moved("write-frames-fp8", "write", 12, 128, 64, "fp8", "32760", "32760"),
        # prompts back from the cache for a layer that reads them whole
        _moved("read-prompts-fp8", "read", 8, 128, 16, "fp8", _spread(16, 5, 512), _spread(16, 5, 512)),
        # a 40-head model's stream of 75,600 tokens back, all frames but the first 21 x 45
        _moved("read-stream-int8", "read", 40, 128, 256, "int8", "75600", "74655"),
        # the first tokens of a few short sequences: latency
        _decode("decode-short-int8", 16, 4, 64, 16, "int8", "1,33,129,300"),
        # one sequence of the length of a video's latent grid and one token
        _decode("decode-one-long-fp8", 12, 12, 128, 64, "fp8", "32761"),
        # a server's batch, lengths from a few tokens to thousands, grouped heads
        _decode("decode-batch", 40, 8, 128, 64, "none", _spread(64, 17, 8192)),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _heads(rng):
    kv, group = rng.choice([(12, 1), (16, 1), (1, 8), (2, 7), (4, 4), (8, 3), (8, 5), (8, 8), (3, 16), (5, 1), (2, 20)])
    return kv * group, kv


def draw(rng):
    """Up to 5.8e11 operations of packed attention, 2e8 elements of its queries, 2e8 of a cache's keys."""
    kind, d = rng.choice(["packed", "packed", "packed_bwd", "packed_bwd", "write", "read", "decode", "decode"]), rng.choice([64, 128])
    H, H_kv = _heads(rng)
    n = rng.choice([1, 1, 2, 3, 5, 8, 24])
    if kind.startswith("packed"):
        form, causal = rng.choice(["self", "self", "prompt", "past"]), rng.random() < 0.5
        pairs = 5.8e11 / (d * H * (10 if kind == "packed_bwd" else 4))
        side = 2.5e9 / H                                           # product of the two sums of lengths
        if form == "prompt":
            k = [rng.choice([0, 1, 77, rng.randint(2, 600)]) if n > 1 else rng.randint(1, 600) for _ in range(n)]
            most = max(4, min(40000, int(min(pairs, side) / (n * max(1, sum(k)))), int(2e8 / (n * H * d))))
            q, causal = [_log_int(rng, max(1, most // 16), most) for _ in range(n)], False
        elif form == "past":
            most = max(8, min(20000, int(min(pairs / n, side / (n * n)) / 64)))
            k = [_log_int(rng, 4, most) for _ in range(n)]
            q = [min(x, rng.randint(1, 64)) for x in k]
        else:
            most = max(4, min(6000, int(math.sqrt(min(pairs / n, side / (n * n))))))
            q = [_log_int(rng, max(1, most // 32), most) for _ in range(n)]
            k = list(q)
        c = _packed("", kind, H, H_kv, d, _text(q), _text(k), causal, rng.random() < 0.5)
    else:
        n = rng.choice([1, 1, 3, 8, 33, 96])
        quant, page = rng.choice(["none", "fp8", "int8"]), rng.choice([16, 32, 64, 128, 256])
        most = max(32, min(75601 if n < 9 else 9000, int(2e8 / (n * H_kv * d))))
        lengths = [_log_int(rng, 1, most) if n > 1 else _log_int(rng, most // 16 + 1, most) for _ in range(n)]
        if kind == "decode":
            c = _decode("", H, H_kv, d, page, quant, _text(lengths))
        else:
            form = rng.choice(["one", "all", "some"])
            new = [1 if form == "one" else x if form == "all" else rng.randint(0, x) for x in lengths]
            new[0] = max(1, new[0])
            c = _moved("", kind, H_kv, d, page, quant, _text(lengths), _text(new))
    del c["name"]
    return c


def _ints(text):
    return [int(t) for t in text.split(",")]


def _starts(lengths):
    """0 and the running sum, int32 on the GPU."""
    s = [0]
    for n in lengths:
        s.append(s[-1] + n)
    return torch.tensor(s, dtype=torch.int32, device="cuda")


def _normal(gen, shape, by=1.0):
    """Normal values whose spread differs from channel to channel, as activations of a trained model have it; bf16."""
    x = torch.randn(shape, generator=gen, device="cuda")
    x *= by * torch.exp(0.4 * torch.randn(shape[-1], generator=gen, device="cuda"))
    return x.to(torch.bfloat16)


def _keys_values(gen, tokens, heads, d, joint):
    if joint:
        t = _normal(gen, (tokens, 3, heads, d))
        return t[:, 1], t[:, 2]
    return _normal(gen, (tokens, heads, d)), _normal(gen, (tokens, heads, d))


def _prepare_packed(case, gen):
    H, H_kv, d, nq, nk = case["H"], case["H_kv"], case["d"], _ints(case["q"]), _ints(case["k"])
    s = {"case": case, "q_start": _starts(nq), "k_start": _starts(nk)}
    s["q"] = _normal(gen, (sum(nq), H, d))
    s["k"], s["v"] = _keys_values(gen, sum(nk), H_kv, d, case["joint"])
    if case["kind"] == "packed_bwd":
        s["dout"] = _normal(gen, (sum(nq), H, d), 0.1)
        out, s["lse"] = _attend(s)                                 # what the forward pass kept
        s["out"] = out.to(torch.bfloat16)
        s["dq"] = torch.empty_like(s["q"])
        t = torch.empty((sum(nk), 3, H_kv, d) if case["joint"] else (3, sum(nk), H_kv, d), dtype=torch.bfloat16, device="cuda")
        s["dk"], s["dv"] = (t[:, 1], t[:, 2]) if case["joint"] else (t[1], t[2])
    else:
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((H, sum(nq)), device="cuda")
    if own:
        from paper_2602_12675_amd import api
        s["params"] = api.make_packed_params(len(nq), sum(nq), sum(nk), H, H_kv, d, causal=case["causal"],
                                             kv_stride=(d, 3 * H_kv * d) if case["joint"] else None)
        s["workspace"] = torch.empty(api.sla2_packed_workspace_bytes(s["params"], case["kind"] == "packed_bwd"), dtype=torch.uint8, device="cuda")
    return s


STORED = {"none": torch.bfloat16, "fp8": torch.float8_e4m3fn, "int8": torch.int8}
TOP = {"fp8": 448.0, "int8": 127.0}


def _prepare_cache(case, gen):
    H_kv, d, page, lengths = case["H_kv"], case["d"], case["page"], _ints(case["lengths"])
    s = {"case": case, "length": torch.tensor(lengths, dtype=torch.int32, device="cuda")}
    need = [-(-n // page) for n in lengths]
    wide, pages = max(need), sum(need) + 3
    ids = torch.randperm(pages, generator=gen, device="cuda")[:sum(need)].int()
    table, at = torch.zeros((len(lengths), wide), dtype=torch.int32, device="cuda"), 0
    for b, n in enumerate(need):                                   # pages behind a sequence's last one: 0, not read
        table[b, :n] = ids[at:at + n]
        at += n
    s["table"] = table
    shape = (pages, H_kv, page, d)
    if case["kind"] == "write":
        s["k_cache"], s["v_cache"] = (torch.zeros(shape, dtype=STORED[case["quant"]], device="cuda") for _ in range(2))
        if case["quant"] != "none":
            s["k_scale"], s["v_scale"] = (torch.zeros(shape[:3], device="cuda") for _ in range(2))
    else:
        for x in ("k", "v"):
            codes, scale = _coded(case["quant"], _normal(gen, shape))
            s[x + "_cache"] = codes
            if scale is not None:
                s[x + "_scale"] = scale
    if case["kind"] == "decode":
        s["q"] = _normal(gen, (len(lengths), case["H"], d))
        s["out"] = torch.empty_like(s["q"])
        rows = 0
    else:
        new = _ints(case["new"])
        rows = sum(new)
        s["start"] = _starts(new)
        s["first"] = torch.tensor([a - b for a, b in zip(lengths, new)], dtype=torch.int32, device="cuda")
        if case["kind"] == "write":
            s["k"], s["v"] = _keys_values(gen, rows, H_kv, d, True)
        else:
            s["k"], s["v"] = (torch.empty((rows, H_kv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    if own:
        from paper_2602_12675_amd import api
        s["params"] = api.make_cache_params(
            len(lengths), case.get("H", H_kv), H_kv, d, pages, page, wide, tokens=rows,
            quant_mode={"none": api.SLA2_QUANT_NONE, "fp8": api.SLA2_QUANT_FP8, "int8": api.SLA2_QUANT_INT8}[case["quant"]],
            kv_stride=(d, 3 * H_kv * d) if case["kind"] == "write" else None)
        if case["kind"] == "decode":
            s["workspace"] = torch.empty(api.sla2_cache_workspace_bytes(s["params"]), dtype=torch.uint8, device="cuda")
    return s


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (_prepare_packed if case["kind"].startswith("packed") else _prepare_cache)(case, gen)


# ---- the plain forms: elementary operations in 32 bits ----

def _sequence(start, rows):
    """The sequence of each row."""
    return (torch.arange(rows, device="cuda")[:, None] >= start[None, 1:]).sum(1)


def _grouped(s, x):
    """[tokens, H_kv, d] -> [H, tokens, d] in 32 bits: every query head's keys or values."""
    return x.float().repeat_interleave(s["case"]["H"] // s["case"]["H_kv"], 1).transpose(0, 1)


def _scores(s):
    """[H, queries, keys]: q . k / sqrt(d), -inf where a query does not read a key."""
    case, q, k = s["case"], s["q"].float().transpose(0, 1), _grouped(s, s["k"])
    sq, sk = _sequence(s["q_start"], q.shape[1]), _sequence(s["k_start"], k.shape[1])
    reads = sq[:, None] == sk[None]
    if case["causal"]:
        # place in its sequence, counted from the sequence's end
        i = torch.arange(q.shape[1], device="cuda") - s["q_start"][sq + 1]
        j = torch.arange(k.shape[1], device="cuda") - s["k_start"][sk + 1]
        reads = reads & (j[None] <= i[:, None])
    t = q @ k.transpose(1, 2)
    return t.mul_(case["d"] ** -0.5).masked_fill_(~reads, -math.inf)


def _softmax(t):
    """(exp(t - m) in place of t, its sums, the logarithm of the sum of exp(t)); a row of -inf gives zeros and -inf."""
    m = t.amax(-1, keepdim=True).clamp_min(-3e38)
    p = t.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    return p, total, torch.where(total > 0, m + total.log(), -math.inf)[..., 0]


def _attend(s):
    """(out [queries, H, d], lse [H, queries]) in 32 bits"""
    p, total, lse = _softmax(_scores(s))
    out = p @ _grouped(s, s["v"]) / total.clamp_min(1e-38)
    return out.transpose(0, 1), lse


def _plain_packed(s):
    out, lse = _attend(s)
    return {"out": out.to(torch.bfloat16), "lse": lse}


def _plain_packed_bwd(s):
    case = s["case"]
    H_kv, d = case["H_kv"], case["d"]
    # a row that reads no key has lse = -inf, and all of its scores are -inf too
    p = _scores(s).sub_(s["lse"].clamp_min(-3e38)[..., None]).exp_()
    g = s["dout"].float().transpose(0, 1)
    delta = (g * s["out"].float().transpose(0, 1)).sum(-1, keepdim=True)

    def shared(x):                                                 # the sum over the query heads of a key head, [keys, H_kv, d]
        return x.view(H_kv, -1, x.shape[1], d).sum(1).transpose(0, 1).to(torch.bfloat16)

    dv = shared(p.transpose(1, 2) @ g)
    ds = (g @ _grouped(s, s["v"]).transpose(1, 2)).sub_(delta).mul_(p).mul_(d ** -0.5)
    dk = shared(ds.transpose(1, 2) @ s["q"].float().transpose(0, 1))
    dq = (ds @ _grouped(s, s["k"])).transpose(0, 1).to(torch.bfloat16)
    return {"dq": dq, "dk": dk, "dv": dv}


def _coded(quant, x):
    """(codes, scales or None) of rows of bf16 values: one scale a row, its largest magnitude over the code's."""
    if quant == "none":
        return x, None
    x, top = x.float(), TOP[quant]
    amax = x.abs().amax(-1)
    some = amax > 0
    y = x * torch.where(some, top / amax, 1.0)[..., None]
    return (y if quant == "fp8" else y.round()).to(STORED[quant]), torch.where(some, amax / top, 1.0)


def _places(s, rows):
    """(page, slot) of each row that is written or read."""
    b = _sequence(s["start"], rows)
    at = s["first"][b] + torch.arange(rows, device="cuda") - s["start"][b]
    return s["table"][b, at // s["case"]["page"]].long(), at % s["case"]["page"]


def _bits(x):
    return x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x


def _plain_write(s):
    page, slot = _places(s, s["k"].shape[0])
    k, ks = _coded(s["case"]["quant"], s["k"])
    v, vs = _coded(s["case"]["quant"], s["v"])
    _bits(s["k_cache"])[page, :, slot] = _bits(k)
    _bits(s["v_cache"])[page, :, slot] = _bits(v)
    out = {"k": s["k_cache"], "v": s["v_cache"]}
    if ks is None:
        return out
    s["k_scale"][page, :, slot] = ks
    s["v_scale"][page, :, slot] = vs
    return dict(out, k_scale=s["k_scale"], v_scale=s["v_scale"])


def _values(s, x, index):
    """What the cache holds at `index`, in 32 bits."""
    codes = _bits(s[x + "_cache"])[index]
    codes = (codes.view(torch.float8_e4m3fn) if s["case"]["quant"] == "fp8" else codes).float()
    return codes if s["case"]["quant"] == "none" else codes * s[x + "_scale"][index][..., None]


def _plain_read(s):
    page, slot = _places(s, s["k"].shape[0])
    return {x: _values(s, x, (page, slice(None), slot)).to(torch.bfloat16) for x in ("k", "v")}


def _plain_decode(s):
    case = s["case"]
    B, wide = s["table"].shape
    H_kv, d = case["H_kv"], case["d"]
    index = (s["table"].long(),)
    k, v = (_values(s, x, index).transpose(1, 2).reshape(B, H_kv, wide * case["page"], d) for x in ("k", "v"))
    t = s["q"].float().view(B, H_kv, -1, d) @ k.transpose(2, 3) * d ** -0.5
    behind = torch.arange(wide * case["page"], device="cuda") >= s["length"][:, None]
    p, total, _ = _softmax(t.masked_fill_(behind[:, None, None], -math.inf))
    return {"out": (p @ v / total.clamp_min(1e-38)).view(B, -1, d).to(torch.bfloat16)}


# ---- the framework's calls ----

def _own_packed(s):
    from paper_2602_12675_amd import api
    api.sla2_packed_forward(s["params"], s["q"], s["k"], s["v"], s["q_start"], s["k_start"], s["out"], lse=s["lse"], workspace=s["workspace"])
    return {"out": s["out"], "lse": s["lse"]}


def _own_packed_bwd(s):
    from paper_2602_12675_amd import api
    api.sla2_packed_backward(s["params"], s["q"], s["k"], s["v"], s["q_start"], s["k_start"], s["out"], s["lse"], s["dout"], s["dq"],
                             s["dk"], s["dv"], workspace=s["workspace"])
    return {"dq": s["dq"], "dk": s["dk"], "dv": s["dv"]}


def _own_write(s):
    from paper_2602_12675_amd import api
    api.sla2_cache_write(s["params"], s["k"], s["v"], s["table"], s["k_cache"], s["v_cache"], k_scale=s.get("k_scale"),
                         v_scale=s.get("v_scale"), start=s["start"], first=s["first"])
    out = {"k": s["k_cache"], "v": s["v_cache"]}
    return dict(out, k_scale=s["k_scale"], v_scale=s["v_scale"]) if "k_scale" in s else out


def _own_read(s):
    from paper_2602_12675_amd import api
    api.sla2_cache_read(s["params"], s["k_cache"], s["v_cache"], s["table"], s["k"], s["v"], k_scale=s.get("k_scale"),
                        v_scale=s.get("v_scale"), start=s["start"], first=s["first"])
    return {"k": s["k"], "v": s["v"]}


def _own_decode(s):
    from paper_2602_12675_amd import api
    api.sla2_cache_attention(s["params"], s["q"], s["k_cache"], s["v_cache"], s["table"], s["length"], s["out"], k_scale=s.get("k_scale"),
                             v_scale=s.get("v_scale"), workspace=s["workspace"])
    return {"out": s["out"]}


def run(s):
    kind = s["case"]["kind"]
    if own:
        return {"packed": _own_packed, "packed_bwd": _own_packed_bwd, "write": _own_write, "read": _own_read, "decode": _own_decode}[kind](s)
    return {"packed": _plain_packed, "packed_bwd": _plain_packed_bwd, "write": _plain_write, "read": _plain_read,
            "decode": _plain_decode}[kind](s)


def _pairs(case):
    """Pairs of a query and a key that it reads, of one head."""
    n = 0
    for q, k in zip(_ints(case["q"]), _ints(case["k"])):
        if case["causal"]:
            blind = max(0, q - k)                                  # the first queries, which read nothing
            m = q - blind
            n += m * (k - m) + m * (m + 1) // 2
        else:
            n += q * k
    return n


def work(case):
    d, H_kv = case["d"], case["H_kv"]
    if case["kind"].startswith("packed"):
        tq, tk, H = sum(_ints(case["q"])), sum(_ints(case["k"])), case["H"]
        q, kv, row = 2 * tq * H * d, 2 * tk * H_kv * d, 4 * tq * H
        if case["kind"] == "packed":
            return {"bytes": 2 * q + 2 * kv + row, "flops": 4 * d * H * _pairs(case)}
        return {"bytes": 4 * q + 4 * kv + row, "flops": 10 * d * H * _pairs(case)}
    held = {"none": 2 * d, "fp8": d + 4, "int8": d + 4}[case["quant"]]         # of one token and head, with its scale
    if case["kind"] == "decode":
        n, H, B = sum(_ints(case["lengths"])), case["H"], len(_ints(case["lengths"]))
        return {"bytes": 2 * n * H_kv * held + 4 * B * H * d, "flops": 4 * n * H * d}
    rows = sum(_ints(case["new"])) * H_kv * 2                                  # of keys and of values
    return {"bytes": rows * (2 * d + held), "flops": rows * d * (1 if case["quant"] == "none" else 3)}


# ---- the definitions in 64 bits, a sequence after the other; gradients by differentiation ----

def _exact_packed(s):
    case = s["case"]
    group, qs, ks = case["H"] // case["H_kv"], s["q_start"].tolist(), s["k_start"].tolist()
    bwd = case["kind"] == "packed_bwd"
    q, k, v = (s[x].double().requires_grad_(bwd) for x in ("q", "k", "v"))
    outs, lses = [], []
    for a, b, c, e in zip(qs, qs[1:], ks, ks[1:]):
        if e == c:
            outs.append(0.0 * q[a:b])
            lses.append(torch.full((case["H"], b - a), -math.inf, dtype=torch.float64, device="cuda"))
            continue
        kk, vv = (x[c:e].permute(1, 0, 2)[:, None] for x in (k, v))
        t = torch.matmul(q[a:b].permute(1, 0, 2).reshape(case["H_kv"], group, b - a, -1), kk.transpose(-1, -2)) / math.sqrt(case["d"])
        if case["causal"]:
            t = t.masked_fill(torch.ones((b - a, e - c), dtype=torch.bool, device="cuda").triu(1 + (e - c) - (b - a)), -math.inf)
        lse = torch.logsumexp(t, -1, keepdim=True)
        w = torch.exp(t - torch.where(lse == -math.inf, 0.0, lse))
        outs.append(torch.matmul(w, vv).reshape(case["H"], b - a, -1).permute(1, 0, 2))
        lses.append(lse.reshape(case["H"], b - a))
    out = torch.cat(outs)
    if not bwd:
        return {"out": out, "lse": torch.cat(lses, 1)}
    got = torch.autograd.grad(out, (q, k, v), s["dout"].double(), allow_unused=True)
    return {n: torch.zeros_like(x) if g is None else g for n, x, g in zip(("dq", "dk", "dv"), (q, k, v), got)}


def _nearest_e4m3(y):
    """4 significant bits, the last of the smallest numbers being 2^-9; ties to even."""
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp_min(2.0 ** -6))) - 3)
    return torch.round(y / step) * step


def _tokens(s, b, n):
    """Rows of the cache, (page, slot) of the first n tokens of sequence b."""
    at = torch.arange(n, device="cuda")
    return s["table"][b].long()[at // s["case"]["page"]], at % s["case"]["page"]


def _exact_moved(s):
    case, quant = s["case"], s["case"]["quant"]
    out = {}
    starts, first = s["start"].tolist(), s["first"].tolist()
    for x in ("k", "v"):
        if case["kind"] == "write":
            y = s[x].double()
            amax = y.abs().amax(-1)
            cache = torch.zeros(s[x + "_cache"].shape, dtype=torch.float64, device="cuda")
            scale = torch.zeros(cache.shape[:3], dtype=torch.float64, device="cuda")
            if quant != "none":
                unit = torch.where(amax > 0, amax / TOP[quant], 1.0)
                y = _nearest_e4m3(y / unit[..., None])
        else:
            got = torch.zeros(s[x].shape, dtype=torch.float64, device="cuda")
        for b in range(len(first)):
            n = starts[b + 1] - starts[b]
            page, slot = (t[first[b]:] for t in _tokens(s, b, first[b] + n))
            if case["kind"] == "write":
                cache[page, :, slot] = y[starts[b]:starts[b + 1]]
                if quant != "none":
                    scale[page, :, slot] = unit[starts[b]:starts[b + 1]]
            else:
                t = _bits(s[x + "_cache"])[page, :, slot]
                t = (t.view(torch.float8_e4m3fn) if quant == "fp8" else t).double()
                got[starts[b]:starts[b + 1]] = t if quant == "none" else t * s[x + "_scale"].double()[page, :, slot][..., None]
        if case["kind"] == "write":
            out[x] = None if quant == "int8" else cache            # whole numbers: the two sides' have to be equal
            if quant != "none":
                out[x + "_scale"] = scale
        else:
            out[x] = got
    return out


def _exact_decode(s):
    case, rows = s["case"], []
    for b, n in enumerate(s["length"].tolist()):
        page, slot = _tokens(s, b, n)
        kv = []
        for x in ("k", "v"):
            t = _bits(s[x + "_cache"])[page, :, slot]
            t = (t.view(torch.float8_e4m3fn) if case["quant"] == "fp8" else t).double()
            kv.append((t if case["quant"] == "none" else t * s[x + "_scale"].double()[page, :, slot][..., None]).permute(1, 0, 2))
        t = torch.matmul(s["q"][b].double().view(case["H_kv"], -1, case["d"]), kv[0].transpose(1, 2)) / math.sqrt(case["d"])
        rows.append(torch.matmul(torch.softmax(t, -1), kv[1]).reshape(case["H"], case["d"]))
    return {"out": torch.stack(rows)}


def exact(case, seed):
    s = prepare(case, seed)
    return (_exact_packed if case["kind"].startswith("packed") else _exact_decode if case["kind"] == "decode" else _exact_moved)(s)
