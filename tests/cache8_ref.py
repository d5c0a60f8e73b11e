"""Plain forms of the operators over 8-bit paged caches, and random caches to run them on (host side, numpy)."""
import numpy as np
import torch

import paged_ref as ref

LOWEST = -100
NAN = 0x7F


def e4m3(y):
    """y (64 bits, |y| <= 448 but for a rounding) to the nearest e4m3 number, ties to even, as numbers; what is not finite:
    not a number."""
    y = np.asarray(y, np.float64)
    with np.errstate(all="ignore"):
        step = np.exp2(np.maximum(np.floor(np.log2(np.maximum(np.abs(y), 2.0 ** -40))), -6) - 3)
        z = np.clip(np.rint(y / step) * step, -448, 448)
    return np.where(np.isfinite(y), z, np.nan)


def to_bytes(x):
    """The bytes of e4m3 numbers: the table of all 256, looked up (the sign of a zero is its own)."""
    table = numbers(np.arange(127, dtype=np.uint8))
    at = np.searchsorted(table, np.abs(np.where(np.isnan(x), 0, x)))
    assert np.array_equal(table[at], np.abs(np.where(np.isnan(x), 0, x)))
    return np.where(np.isnan(x), NAN, at + 128 * np.signbit(x)).astype(np.uint8)


def numbers(b):
    """The numbers of e4m3 bytes: sign, four bits of exponent (bias 7), three of mantissa; 0x7F and 0xFF: not a number."""
    b = np.asarray(b).astype(np.int64)
    e, m = b >> 3 & 15, b & 7
    x = np.where(e == 0, m * 2.0 ** -9, (8 + m) * np.exp2(e - 10.0))
    return np.where((b & 0x7F) == NAN, np.nan, np.where(b >= 128, -x, x))


def scale_for(top):
    """The smallest power of two from 2^LOWEST on of which top is at most 448 times."""
    e = LOWEST
    with np.errstate(divide="ignore"):
        e = np.maximum(np.floor(np.log2(np.asarray(top, np.float64) / 448)) - 1, LOWEST)
    while np.any(top > 448 * np.exp2(e)):
        e = np.where(top > 448 * np.exp2(e), e + 1, e)
    return np.exp2(e)


def make_cache(rng, lens, Hkv, D, P, spare=0, spoil=True, powers=True):
    """Host dict of a random cache: bytes, scales from 2^-12 to 2^-3 (any in that range without `powers`); rows past the live
    ones are not numbers with `spoil`."""
    c = ref.make_cache(rng, lens, Hkv, D, P, spare=spare, spoil=False)
    nb = len(c["k"])
    for x in ("k", "v"):
        b = to_bytes(e4m3(rng.normal(0, 60, size=(nb, Hkv, P, D))))
        if spoil:
            live = np.zeros(nb, np.int64)
            for s, n in enumerate(lens):
                for j in range(c["table"].shape[1]):
                    if c["table"][s, j] >= 0:
                        live[c["table"][s, j]] = min(P, max(0, n - j * P))
            for i in range(nb):
                b[i, :, live[i]:] = NAN
        c[x] = b
    e = rng.uniform(-12, -3, size=(nb, Hkv, 2))
    c["scale"] = np.exp2(np.rint(e) if powers else e).astype(np.float32)
    return c


def values(c):
    """The cache with the numbers that it stands for (fp32 products: exact where scales are powers of two)."""
    out = dict(c)
    for i, x in enumerate(("k", "v")):
        out[x] = torch.from_numpy(numbers(c[x]) * c["scale"][:, :, i, None, None].astype(np.float64))
    return out




def check_attention(c, q, got, lse=None, **kw):
    """paged_ref's check over the numbers that the cache stands for, in 64 bits."""
    v = values(c)
    f64 = ref.f64
    try:
        ref.f64 = lambda t: t.detach().cpu().numpy().astype(np.float64) if t.dtype == torch.float64 else f64(t)
        ref.check_attention(v, q, got, lse, **kw)
    finally:
        ref.f64 = f64


def to_device(c, summary=None):
    import paper_2601_08670_gb300 as pced
    t = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return pced.PagedCache8(t(c["k"]).view(torch.float8_e4m3fn), t(c["v"]).view(torch.float8_e4m3fn), t(c["scale"]),
                            t(c["table"]), t(c["lens"]), summary=None if summary is None else t(summary),
                            key_step=t(c["key_step"]))


def rotated32(x, rope):
    """Rotate-half of x [T, H, D] (fp32) by table rows [T, D], every product and sum rounded to fp32."""
    D = x.shape[2]
    co, si = rope[:, None, :D // 2].astype(np.float32), rope[:, None, D // 2:].astype(np.float32)
    a, b = x[..., :D // 2], x[..., D // 2:]
    return np.concatenate([a * co - b * si, b * co + a * si], axis=2)


def append(c, k, v, new, summary=None):
    """(cache, summary) after the new rows k, v (fp32 [T, Hkv, D], rotated) of the sequences, new[s] each; the definition,
    with its fp32 roundings."""
    out = {x: c[x].copy() for x in ("k", "v", "scale")}
    summary = None if summary is None else summary.copy()
    P, t = c["P"], 0
    for s, (n, m) in enumerate(zip(c["lens"], new)):
        row = int(n) - m
        while row < n:
            j, at = row // P, row % P
            here = min(P - at, int(n) - row)
            b = c["table"][s, j]
            for i, (name, x) in enumerate((("k", k), ("v", v))):
                x = x[t:t + here].transpose(1, 0, 2).astype(np.float32)  # [Hkv, here, D]
                top = np.where(np.isfinite(x), np.abs(x), 0).max(axis=(1, 2))
                s0 = out["scale"][b, :, i]
                need = scale_for(top).astype(np.float32)
                now = need if at == 0 else np.fmax(s0, need)
                with np.errstate(all="ignore"):
                    inv, ratio = np.float32(1) / now, s0 / now
                    out[name][b, :, at:at + here] = to_bytes(e4m3(x * inv[:, None, None]))
                    moved = to_bytes(e4m3(numbers(out[name][b, :, :at]).astype(np.float32) * ratio[:, None, None]))
                out[name][b, :, :at] = np.where((now == s0)[:, None, None], out[name][b, :, :at], moved)
                out["scale"][b, :, i] = now
            if summary is not None:
                for h in range(c["Hkv"]):
                    w = ref.bounds(k[t:t + here, h], c["key_step"][h])
                    summary[b, h] = w if at == 0 else np.stack([np.maximum(w[0], summary[b, h, 0]),
                                                                np.minimum(w[1], summary[b, h, 1])])
            row, t = row + here, t + here
    return dict(c, **out), summary
