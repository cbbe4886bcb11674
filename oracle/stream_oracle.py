"""fp64 statement of attention over packed sequences, its gradients, and a paged cache of keys and values (sla2_packed_*, sla2_cache_*).

One sequence and head at a time, scores written out.  Test infrastructure only; it shares no code with the HIP path.  Beside its values
each function returns what bounds on a rounded computation are made of: `mag`, sums of the absolute values of a result's terms."""
import numpy as np

import sla2_oracle as O

TOP = {"fp8": np.float32(448.0), "int8": np.float32(127.0)}


def bounds(start, tokens):
    """(first, count) of every sequence, whatever the offsets hold inside 0 .. tokens."""
    a = np.clip(np.asarray(start[:-1], dtype=np.int64), 0, tokens)
    b = np.clip(np.asarray(start[1:], dtype=np.int64), a, tokens)
    return list(zip(a.tolist(), (b - a).tolist()))


def reads(nq, nk, causal):
    """[nq, nk]: whether a query reads a key"""
    if not causal:
        return np.ones((nq, nk), dtype=bool)
    return np.arange(nk)[None] <= np.arange(nq)[:, None] + (nk - nq)


def attend(q, k, v, mask, scale):
    """q [nq, d], k, v [nk, d], all fp64 -> out, lse, mag (sum p |v|), smag (largest scale sum |q k| of a row's keys)"""
    nq, nk = mask.shape
    s = scale * (q @ k.T)
    smag = np.where(mask, scale * (np.abs(q) @ np.abs(k).T), 0.0).max(1, initial=0.0)
    out, mag, lse = np.zeros_like(q), np.zeros_like(q), np.full(nq, -np.inf)
    for i in range(nq):
        j = mask[i]
        if not j.any():
            continue
        m = s[i, j].max()
        p = np.exp(s[i, j] - m)
        lse[i] = m + np.log(p.sum())
        p /= p.sum()
        out[i], mag[i] = p @ v[j], p @ np.abs(v[j])
    return out, lse, mag, smag


def packed_forward(q, k, v, q_start, k_start, causal, scale):
    """q [Tq, H, d], k, v [Tk, H_kv, d] -> dict(out, lse [H, Tq], mag, smag [H, Tq]); NaN where no sequence is"""
    Tq, H, d = q.shape
    group = H // k.shape[1]
    r = dict(out=np.full(q.shape, np.nan), mag=np.full(q.shape, np.nan), lse=np.full((H, Tq), np.nan), smag=np.full((H, Tq), np.nan))
    for (a, nq), (c, nk) in zip(bounds(q_start, Tq), bounds(k_start, k.shape[0])):
        for h in range(H):
            rows = slice(a, a + nq)
            r["out"][rows, h], r["lse"][h, rows], r["mag"][rows, h], r["smag"][h, rows] = attend(
                q[rows, h], k[c:c + nk, h // group], v[c:c + nk, h // group], reads(nq, nk, causal), scale)
    return r


def packed_backward(q, k, v, q_start, k_start, causal, scale, out, lse, dout):
    """Gradients for the stored out and lse: P = exp(S - lse), D = rowsum(dO . O), dS = P (dO V^T - D); with the sums that bounds need:
    dq_mag etc. hold sum |dS| |k| .., dq_small etc. sum p (sum |dO v| + sum |dO o|) |k| .. (what fp32 rounding in dP and D acts on)."""
    Tq, H, d = q.shape
    group, Tk = H // k.shape[1], k.shape[0]
    r = {n: np.zeros(s) for n, s in (("dq", q.shape), ("dk", k.shape), ("dv", k.shape), ("dq_mag", q.shape), ("dk_mag", k.shape),
                                     ("dv_mag", k.shape), ("dq_small", q.shape), ("dk_small", k.shape))}
    r["smag"] = 0.0
    for (a, nq), (c, nk) in zip(bounds(q_start, Tq), bounds(k_start, Tk)):
        mask = reads(nq, nk, causal)
        for h in range(H):
            i, j, hk = slice(a, a + nq), slice(c, c + nk), h // group
            qq, kk, vv, g, o = q[i, h], k[j, hk], v[j, hk], dout[i, h], out[i, h]
            L = lse[h, i][:, None]
            s = scale * (qq @ kk.T)
            p = np.where(mask & np.isfinite(L), np.exp(np.where(mask & np.isfinite(L), s - np.where(np.isfinite(L), L, 0.0), -np.inf)), 0.0)
            D = (g * o).sum(1, keepdims=True)
            ds = p * (g @ vv.T - D)
            small = p * (np.abs(g) @ np.abs(vv).T + (np.abs(g) * np.abs(o)).sum(1, keepdims=True))
            r["dq"][i, h] = scale * ds @ kk
            r["dq_mag"][i, h] = scale * np.abs(ds) @ np.abs(kk)
            r["dq_small"][i, h] = scale * small @ np.abs(kk)
            r["dk"][j, hk] += scale * ds.T @ qq
            r["dk_mag"][j, hk] += scale * np.abs(ds).T @ np.abs(qq)
            r["dk_small"][j, hk] += scale * small.T @ np.abs(qq)
            r["dv"][j, hk] += p.T @ g
            r["dv_mag"][j, hk] += p.T @ np.abs(g)
            if nq and nk:
                r["smag"] = max(r["smag"], float((scale * (np.abs(qq) @ np.abs(kk).T) * mask).max()), float(np.abs(np.where(np.isfinite(L), L, 0)).max()))
    return r


def code_rows(x, quant):
    """x [..., d] float32 -> (values of the codes as float32, scales float32); the decisions are those of fp32"""
    top = TOP[quant]
    fine = np.isfinite(x).all(-1)
    amax = np.where(fine, np.abs(np.where(np.isfinite(x), x, 0)).max(-1), 0).astype(np.float32)
    some = amax >= np.float32(2.0 ** -100)
    by = np.where(some, top * (np.float32(1) / np.where(some, amax, np.float32(1))), 0).astype(np.float32)
    y = (np.where(np.isfinite(x), x, 0).astype(np.float32) * by[..., None]).astype(np.float32)
    codes = O.e4m3_round(y.astype(np.float64)).astype(np.float32) if quant == "fp8" else np.rint(y)
    scale = np.where(some, (np.where(some, amax, np.float32(1)) * (np.float32(1) / top)).astype(np.float32), np.float32(1.0))
    return np.where(fine[..., None], codes, 0).astype(np.float32), np.where(fine, scale, np.float32(np.nan)).astype(np.float32)


def place(b, t, table, page_size, pages):
    """(page, slot) of token t of sequence b, None if it has none"""
    if t < 0 or t >= table.shape[1] * page_size:
        return None
    page = int(table[b, t // page_size])
    return (page, t % page_size) if 0 <= page < pages else None


def rows_of(start, first, tokens, B):
    """(row, sequence, token) of every row that is of a sequence"""
    for b in range(B):
        lo, hi = (b, b + 1) if start is None else (int(start[b]), int(start[b + 1]))
        for i in range(max(lo, 0), min(hi, tokens)):
            yield i, b, i - lo + (0 if first is None else int(first[b]))
