"""Plain 64-bit forms of the operators over paged caches, and random caches to
run them on (host side, numpy)."""
import math

import numpy as np
import torch


def rng_bf16(rng, shape, sigma=1.0):
    return torch.from_numpy(rng.normal(0.0, sigma, size=shape).astype(np.float32)).to(torch.bfloat16)


def make_table(rng, lens, P, spare=0, extra_blocks=3):
    """(table [S, max_blocks], pool blocks): scattered blocks for max(lens, 1) + spare rows each, -1 after them."""
    need = [(max(n, 1) + spare + P - 1) // P for n in lens]
    order = rng.permutation(sum(need) + extra_blocks)
    table = np.full((len(lens), max(need) + 1), -1, np.int32)
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = order[at:at + n]
        at += n
    return table, sum(need) + extra_blocks


def make_cache(rng, lens, Hkv, D, P, spare=0, spoil=True, sigma=1.0):
    """Host dict of a random cache; rows past the live ones are not numbers with `spoil`."""
    table, nb = make_table(rng, lens, P, spare)
    k, v = rng_bf16(rng, (nb, Hkv, P, D), sigma), rng_bf16(rng, (nb, Hkv, P, D), sigma)
    if spoil:
        live = np.zeros(nb, np.int64)
        for s, n in enumerate(lens):
            for j in range(table.shape[1]):
                if table[s, j] >= 0:
                    live[table[s, j]] = min(P, max(0, n - j * P))
        for b in range(nb):
            k[b, :, live[b]:] = float("nan")
            v[b, :, live[b]:] = float("inf")
    return dict(table=table, k=k, v=v, lens=np.asarray(lens, np.int32), P=P, Hkv=Hkv, D=D,
                key_step=(rng.uniform(2.0, 5.0, size=Hkv) / 127).astype(np.float32))


def to_device(c, summary=None):
    import paper_2601_08670_gb300 as pced
    t = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return pced.PagedCache(c["k"].cuda(), c["v"].cuda(), t(c["table"]), t(c["lens"]),
                           summary=None if summary is None else t(summary), key_step=t(c["key_step"]))


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def rows_of(c, s, h, rows):
    """(K, V) in 64 bits of some rows of a sequence."""
    b = c["table"][s, rows // c["P"]]
    return f64(c["k"])[b, h, rows % c["P"]], f64(c["v"])[b, h, rows % c["P"]]


def attention(c, q, sel=None, scale=None):
    """(out, lse, tolerance of out, tolerance of lse), all 64-bit: out [S, Hq, D], the others [S, Hq].

    The tolerances bound fp32 arithmetic: a score is a sum of D products (error at most e = D 2^-24 sum |q k| scale);
    probabilities are held to 16 bits (2^-16), n of them are summed in fp32 (n 2^-24, numerator and denominator), and
    a few roundings of exp2 and the final quotient stay below 2^-20."""
    kf, vf, qf = f64(c["k"]), f64(c["v"]), f64(q)
    S, Hq, D = qf.shape
    Hkv, P = c["Hkv"], c["P"]
    G = Hq // Hkv
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    out, lse = np.zeros((S, Hq, D)), np.full((S, Hq), -np.inf)
    tol_o, tol_l = np.zeros((S, Hq)), np.zeros((S, Hq))
    for s in range(S):
        n = int(c["lens"][s])
        for h in range(Hkv):
            rows = np.arange(n)
            if sel is not None:
                keep = np.asarray(sel[s, h])
                rows = rows[np.isin(rows // P, keep[keep >= 0])]
            if not len(rows):
                continue
            b = c["table"][s, rows // P]
            k, v = kf[b, h, rows % P], vf[b, h, rows % P]
            for g in range(h * G, (h + 1) * G):
                z = k @ qf[s, g] * scale
                m = z.max()
                p = np.exp(z - m)
                out[s, g] = p @ v / p.sum()
                lse[s, g] = m + np.log(p.sum())
                e = D * 2.0 ** -24 * (np.abs(k) @ np.abs(qf[s, g])).max() * abs(scale) + 2.0 ** -22 * np.abs(z).max()
                tol_o[s, g] = np.abs(v).max() * (2 * e + 2.0 ** -16 + len(rows) * 2.0 ** -23 + 2.0 ** -20)
                tol_l[s, g] = e + len(rows) * 2.0 ** -24 + 2.0 ** -20 * max(1.0, abs(lse[s, g]))
    return out, lse, tol_o, tol_l


def check_attention(c, q, got, got_lse=None, sel=None, scale=None, bf16=False):
    out, lse, tol_o, tol_l = attention(c, q, sel, scale)
    got = f64(got)
    assert np.all(np.isfinite(got))
    err = np.abs(got - out) - (2.0 ** -8 * np.abs(out) if bf16 else 0.0)
    assert np.all(err.max(axis=2) <= tol_o), (err.max(axis=2) / np.maximum(tol_o, 1e-30)).max()
    if got_lse is not None:
        got_lse = got_lse.cpu().numpy().astype(np.float64)
        empty = np.isneginf(lse)
        assert np.array_equal(np.isneginf(got_lse), empty)
        assert np.all(np.abs(got_lse - lse)[~empty] <= tol_l[~empty])


def bounds(keys, step):
    """int8 [2, D] of keys [n, D] (fp32 values of the stored bf16): the definition, rounding included."""
    x = keys.astype(np.float32) * (np.float32(1) / np.float32(step))
    hi = np.where(np.isnan(x), 127, np.clip(np.ceil(x), -127, 127)).max(axis=0)
    lo = np.where(np.isnan(x), -127, np.clip(np.floor(x), -127, 127)).min(axis=0)
    return np.stack([hi, lo]).astype(np.int8)


def summaries(c, out):
    """All live blocks' summaries written over a copy of `out` (int8 [num_blocks, Hkv, 2, D])."""
    out = out.copy()
    k = c["k"].float().cpu().numpy()
    for s, n in enumerate(c["lens"]):
        for j in range((int(n) + c["P"] - 1) // c["P"]):
            b = c["table"][s, j]
            for h in range(c["Hkv"]):
                out[b, h] = bounds(k[b, h, :n - j * c["P"]], c["key_step"][h])
    return out


def select(c, summary, q, n_sel, n_first, n_last):
    """The chosen blocks, in whole numbers (a bad table entry scores below all others)."""
    qf = q.float().cpu().numpy()
    S, Hq, D = qf.shape
    Hkv, P = c["Hkv"], c["P"]
    G = Hq // Hkv
    sel = np.full((S, Hkv, n_sel), -1, np.int32)
    for s, n in enumerate(c["lens"]):
        nb = (int(n) + P - 1) // P
        for h in range(Hkv):
            pooled = np.zeros((2, D), np.float32)
            for g in range(G):
                x = qf[s, h * G + g]
                with np.errstate(invalid="ignore"):
                    pooled = pooled + np.stack([np.maximum(x, 0), np.minimum(x, 0)])
            m = np.abs(pooled).max()
            steps = np.zeros((2, D), np.int64)
            if m > 0 and np.isfinite(m):
                steps = np.rint(pooled * (np.float32(127) / m)).astype(np.int64)
            score = np.full(nb, -(1 << 40), np.int64)
            for j in range(nb):
                b = c["table"][s, j]
                if 0 <= b < len(summary):
                    score[j] = (steps * summary[b, h].astype(np.int64)).sum()
                if j < n_first or j >= nb - n_last:
                    score[j] = 1 << 40
            best = np.lexsort((np.arange(nb), -score))[:n_sel]
            sel[s, h, :len(best)] = np.sort(best)
    return sel


def rotate(x, rope):
    """Rotate-half of x [T, H, D] (64 bits) by table rows [T, D]."""
    D = x.shape[2]
    co, si = rope[:, None, :D // 2], rope[:, None, D // 2:]
    a, b = x[..., :D // 2], x[..., D // 2:]
    return np.concatenate([a * co - b * si, b * co + a * si], axis=2)


def process(x, R, history=None, history_len=None, penalties=None, bias_ids=None, bias=None, mask=None, mask_row=None):
    """Logits processed in 64 bits, and the magnitude that the roundings are relative to."""
    y = x.astype(np.float64)
    mag = np.abs(np.where(np.isfinite(y), y, 0.0))
    B, V = len(y) // R, y.shape[1]
    for b in range(B):
        rows = slice(b * R, (b + 1) * R)
        if history is not None:
            toks = [t for t in history[b, :history_len[b]] if 0 <= t < V]
            rep, freq, pres = penalties[b].astype(np.float64)
            for t, c in zip(*np.unique(toks, return_counts=True)):
                col = y[rows, int(t)]
                col = np.where(col > 0, col / rep, col * rep)
                mag[rows, int(t)] = np.abs(np.where(np.isfinite(col), col, 0)) + abs(c * freq) + abs(pres)
                y[rows, int(t)] = col - (c * freq + pres)
        if bias_ids is not None:
            last = {int(t): float(w) for t, w in zip(bias_ids[b], bias[b]) if 0 <= t < V}
            for t, w in last.items():
                y[rows, t] += w
                mag[rows, t] += abs(w) if np.isfinite(w) else 0
        if mask is not None:
            m = b if mask_row is None else int(mask_row[b])
            if 0 <= m < len(mask):
                bits = np.unpackbits(mask[m].astype("<i4").view(np.uint8), bitorder="little")[:V]
                y[rows][:, bits == 0] = -np.inf
    return y, mag
