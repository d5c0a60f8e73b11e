"""Measured work of decoding over 8-bit paged caches, and of sampling.

Three operators, each with its plain form beside the library's call:

* ``append``  ``kv_append`` over a ``PagedCache8``: new keys and values, rotated on the way, into pages of e4m3 numbers
  with a scale for each block, head and kind; a scale that grows moves the rows that its block holds already;
* ``attn``    ``paged_attention`` over a ``PagedCache8``: one new token per sequence, over all or the selected blocks;
* ``sample``  ``sample``: a token for every row of logits, by temperature, top-k, top-p and min-p, from given random numbers.

Shapes are those of the synthetic workloads and of the tests; the inputs are generated here, from the seed alone.
"""
import math

import numpy as np
import torch

own = False  # True: `run` makes the library's calls; False: the plain forms

ROOM = 64      # rows kept free in every cache for the tokens to come
QUERY = 32     # rows of the question, which every cache holds after its document
TOP = 448.0    # e4m3's largest number
LOWEST = -100  # exponent of the smallest scale
E4M3 = torch.float8_e4m3fn

HEADS = {  # name: (query heads, kv heads, head dim)
    "8/2/64": (8, 2, 64),        # the tiny workload
    "16/2/64": (16, 2, 64),      # eight query heads per kv head
    "32/8/128": (32, 8, 128),    # Llama-3-8B shapes
    "28/4/128": (28, 4, 128),    # Qwen2-7B shapes: seven query heads per kv head
}


# ------------------------------------------------------------------- the cases
def listed():
    return [
        # every sequence's next token, one layer of a Llama-3-8B-shaped decode: the smallest append
        dict(name="append_step", kind="append", heads="32/8/128", S=9, lo=2081, hi=2081, new=1, P=64, idle=0, rope=True,
             summary=True),
        # the question's 32 tokens behind each of 33 documents, most in blocks that hold rows already
        dict(name="append_query", kind="append", heads="28/4/128", S=33, lo=700, hi=4000, new=QUERY, P=128, idle=0,
             rope=True, summary=False),
        # sixteen ragged documents of about 1024 rows encoded in one pass: the largest append
        dict(name="append_docs", kind="append", heads="32/8/128", S=16, lo=256, hi=2048, new=0, P=64, idle=0, rope=True,
             summary=True),
        # the tiny workload's layer: the smallest attention, where launches count
        dict(name="attn_tiny", kind="attn", heads="8/2/64", S=3, lo=257, hi=257, P=64, idle=0, keep=0),
        # one layer over eight documents of 2048 rows and the amateur, all blocks
        dict(name="attn_docs", kind="attn", heads="32/8/128", S=9, lo=2081, hi=2081, P=64, idle=0, keep=0),
        # 64 selected blocks of every document of 16384 rows, seven query heads per kv head
        dict(name="attn_select", kind="attn", heads="28/4/128", S=17, lo=16416, hi=16416, P=64, idle=0, keep=64),
        # one very long cache in small blocks, eight query heads per kv head: the split over a long axis
        dict(name="attn_long", kind="attn", heads="16/2/64", S=1, lo=131_104, hi=131_104, P=16, idle=0, keep=0),
        # sixteen queries' ragged documents at once: the largest layer
        dict(name="attn_batch", kind="attn", heads="32/8/128", S=272, lo=256, hi=2048, P=128, idle=0, keep=0),
        # one answer's next token, a usual top-p: the smallest call
        dict(name="sample_one", kind="sample", rows=1, V=128_256, type="fp32", cut="p", mask=False),
        # nine rows of an unembedding that writes bf16 (logits tie), under a grammar's mask, the fifty best tokens
        dict(name="sample_ties", kind="sample", rows=9, V=151_936, type="bf16", cut="k", mask=True),
        # 64 requests without any cut: the whole distribution
        dict(name="sample_whole", kind="sample", rows=64, V=128_256, type="fp32", cut="none", mask=False),
        # 272 requests with parameters of their own, greedy ones among them: the largest call
        dict(name="sample_batch", kind="sample", rows=272, V=151_936, type="fp32", cut="mixed", mask=False),
    ]


def _log(rng, lo, hi):
    """A whole number spread over the logarithm of [lo, hi]."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["append", "append", "attn", "attn", "attn", "sample", "sample"])
    if kind == "sample":
        return dict(kind=kind, rows=_log(rng, 1, 272), V=_log(rng, 1000, 151_936), type=rng.choice(["fp32", "bf16"]),
                    cut=rng.choice(["none", "k", "p", "kp", "min", "mixed"]), mask=rng.random() < 0.4)
    heads = rng.choice(sorted(HEADS))
    S = _log(rng, 1, 272)
    P = rng.choice([16, 32, 64, 64, 128, 192, 256])
    # rows of a sequence: at most about what the largest listed case of the kind holds
    most = {"append": 18_000, "attn": 300_000}[kind]
    hi = _log(rng, 16, max(32, min(131_072, most // S)))
    lo = rng.choice([hi, max(1, hi // rng.randint(2, 16))])
    c = dict(kind=kind, heads=heads, S=S, lo=lo, hi=hi, P=P, idle=rng.choice([0, 0, 1]) if S > 1 else 0)
    if kind == "append":
        c.update(new=rng.choice([0, 1, 1, 2, QUERY, 100]), rope=rng.random() < 0.8, summary=rng.random() < 0.5)
    else:
        c["keep"] = rng.choice([0, 0, 1]) and _log(rng, 1, 128)
    return c


# ----------------------------------------------------------------- the inputs
def _lengths(c):
    """Live rows of every sequence (a property of the case, not of the seed); idle ones hold none."""
    rng = np.random.default_rng([c["S"], c["lo"], c["hi"]])
    lens = rng.integers(c["lo"], c["hi"], endpoint=True, size=c["S"])
    lens[len(lens) - c["idle"]:] = 0
    return lens


def _new(c, lens):
    """New rows of every sequence."""
    return np.minimum(lens, c["new"]) if c["new"] else lens


def _touched(c, lens):
    """(sequence, block of the sequence) of every block that gets new rows."""
    first, last = (lens - _new(c, lens)) // c["P"], (lens + c["P"] - 1) // c["P"]
    n = np.where(_new(c, lens) > 0, last - first, 0)
    seq = np.repeat(np.arange(len(lens)), n)
    return seq, first[seq] + np.arange(len(seq)) - np.repeat(np.cumsum(n) - n, n)


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(shape, sigma, g, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, sigma, generator=g)


def _dev(a, dtype):
    return torch.as_tensor(np.ascontiguousarray(a), dtype=dtype, device="cuda")


def _pages(lens, P, seed):
    """Block table in which the blocks lie scattered over the pool, as a serving allocator leaves them."""
    nblk = (lens + ROOM + P - 1) // P
    order = np.random.default_rng(seed).permutation(int(nblk.sum()))
    seq = np.repeat(np.arange(len(lens)), nblk)
    table = np.full((len(lens), int(nblk.max())), -1, np.int64)
    table[seq, np.arange(len(seq)) - np.repeat(np.cumsum(nblk) - nblk, nblk)] = order
    return table, int(nblk.sum())


def _live(lens, table, nblocks, P):
    """Live rows of every block of the pool."""
    live = np.zeros(nblocks, np.int64)
    j = np.arange(table.shape[1])
    rows = np.clip(lens[:, None] - j[None] * P, 0, P)
    live[table[table >= 0]] = rows[table >= 0]
    return live


def _rope_table(rows, D, theta=5e5):
    """Rotation table [rows, D]: the cosines, then the sines, of fp32(p * fp32(theta^(-2f/D)))."""
    f = _dev((theta ** (-2.0 * np.arange(D // 2) / D)).astype(np.float32), torch.float32)
    ang = (torch.arange(rows, dtype=torch.float32, device="cuda")[:, None] * f).double()
    return torch.cat([ang.cos(), ang.sin()], dim=1).float()


def _steps(top):
    """The smallest power of two, of exponent LOWEST or more, that `top` is at most TOP times."""
    part, exponent = torch.frexp(top)  # TOP is 7/8 * 2^9
    exponent = torch.where(part <= 0.875, exponent - 9, exponent - 8)
    return torch.ldexp(torch.ones_like(top), torch.where(top > 0, exponent, LOWEST).clamp(min=LOWEST))


def _held(pool, live):
    """A pool of bf16 numbers as e4m3 ones with the scales [blocks, heads] of its live rows; what no sequence has written
    yet is not a number."""
    dead = (torch.arange(pool.shape[2], device="cuda")[None] >= live[:, None])[:, None, :, None]
    scale = _steps(pool.abs().masked_fill_(dead, 0).amax(dim=(2, 3)).float())
    held = (pool.float() / scale[:, :, None, None]).to(E4M3)
    held.view(torch.uint8).masked_fill_(dead, 0x7F)
    return held, scale


def prepare(case, seed):
    if case["kind"] == "sample":
        return _prepare_sample(case, seed)
    Hq, Hkv, D = HEADS[case["heads"]]
    S, P = case["S"], case["P"]
    lens, g = _lengths(case), _gen(seed)
    table, nblocks = _pages(lens, P, seed)
    old = lens - _new(case, lens) if case["kind"] == "append" else lens  # rows that the cache holds before the call
    live = _dev(_live(old, table, nblocks, P), torch.int64)
    st = dict(case=case, lens=_dev(lens, torch.int32), table=_dev(table, torch.int32), host=(lens, table),
              status=torch.zeros(1, dtype=torch.int32, device="cuda"), summary=None, step=None)
    # some channels of the keys are far larger than others
    gain = torch.exp(0.5 * _normal((Hkv, 1, D), 1.0, g, torch.float32)).to(torch.bfloat16)
    st["k"], k_scale = _held(_normal((nblocks, Hkv, P, D), 1.0, g).mul_(gain), live)
    st["v"], v_scale = _held(_normal((nblocks, Hkv, P, D), 1.0, g), live)
    st["scale"] = torch.stack([k_scale, v_scale], dim=2).contiguous()
    if case["kind"] == "append":
        m = _new(case, lens)
        T = int(m.sum())
        qkv = _normal((T, Hq + 2 * Hkv, D), 1.0, g)  # one projection's output
        qkv[:, Hq:Hq + Hkv] *= gain[:, 0]
        seq, block = _touched(case, lens)
        st.update(q=qkv[:, :Hq], nk=qkv[:, Hq:Hq + Hkv], nv=qkv[:, Hq + Hkv:], T=T,
                  q_out=torch.empty((T, Hq, D), dtype=torch.bfloat16, device="cuda"),
                  tok_start=_dev(np.concatenate([[0], np.cumsum(m)]), torch.int32),
                  touched=(_dev(seq, torch.int64), _dev(block, torch.int64)),
                  one=case["new"] == 1 and case["idle"] == 0,
                  rope=_rope_table(max(1, int(lens.max())), D) if case["rope"] else None)
        if case["summary"]:
            spread = torch.randint(60, 100, (nblocks, Hkv, 2, D), device="cuda", generator=g, dtype=torch.int32)
            spread[:, :, 1] *= -1
            st["summary"] = spread.to(torch.int8)
            st["step"] = torch.full((Hkv,), 5.0 / 127.0, device="cuda") * (1 + 0.25 * torch.rand(
                Hkv, device="cuda", generator=g))
    else:
        st.update(q=_normal((S, Hq, D), 1.0, g), sel=_choice(case, lens, g) if case["keep"] else None,
                  out=torch.empty((S, Hq, D), dtype=torch.float32, device="cuda"),
                  lse=torch.empty((S, Hq), dtype=torch.float32, device="cuda"))
    if own:
        import paper_2601_08670_gb300 as pced
        st["cache"] = pced.PagedCache8(st["k"], st["v"], st["scale"], st["table"], st["lens"], summary=st["summary"],
                                       key_step=st["step"])
        if case["kind"] == "attn":
            st["ws"] = pced.workspace(pced.paged_attention_workspace_size(S, Hq, Hkv, D), "cuda")
    return st


def _choice(c, lens, g):
    """`keep` blocks of every (sequence, kv head), the last one among them, in ascending order; -1 after them.  In every
    seventeenth sequence, from the ninth on, one head's choice is empty."""
    Hkv, P, keep = HEADS[c["heads"]][1], c["P"], c["keep"]
    nb = _dev((lens + P - 1) // P, torch.int64)[:, None, None]
    most = max(1, int((lens.max() + P - 1) // P))
    j = torch.arange(most, device="cuda")
    key = torch.rand((c["S"], Hkv, most), device="cuda", generator=g)
    key = torch.where(j >= nb, -1.0, torch.where(j == nb - 1, 2.0, key))
    top = key.topk(min(keep, most), dim=2)
    idx = torch.where(top.values < 0, most, top.indices).sort(dim=2).values
    sel = torch.full((c["S"], Hkv, keep), -1, dtype=torch.int32, device="cuda")
    sel[:, :, :idx.shape[2]] = torch.where(idx == most, -1, idx)
    sel[8::17, 0] = -1
    return sel


def _prepare_sample(c, seed):
    """Logits of some rows far flatter than of others; a request without a cut of a kind has that parameter's neutral value."""
    n, V, g = c["rows"], c["V"], _gen(seed)
    spread = 1.0 + 2.5 * torch.rand((n, 1), device="cuda", generator=g)
    x = _normal((n, V), 1.0, g, torch.float32).mul_(spread)
    if c["mask"]:  # what a grammar allows: about one token in six
        x.masked_fill_(torch.rand((n, V), device="cuda", generator=g) > 1 / 6, -math.inf)
    if c["type"] == "bf16":
        x = x.to(torch.bfloat16)

    def pick(values, default, used):
        at = torch.randint(0, len(values), (n,), device="cuda", generator=g)
        return torch.tensor(values if used else [default] * len(values), device="cuda")[at]

    mixed, cut = c["cut"] == "mixed", c["cut"]
    t = 0.4 + 1.1 * torch.rand(n, device="cuda", generator=g)
    if mixed:
        t[4::17] = 0.0  # greedy requests
    return dict(case=c, x=x, temperature=t,
                top_k=pick([0, 1, 20, 50, 1000] if mixed else [50], 0, mixed or "k" in cut).to(torch.int32),
                top_p=pick([1.0, 0.5, 0.9, 0.95, 0.999] if mixed else [0.9, 0.95], 1.0, mixed or cut in ("p", "kp")),
                min_p=pick([0.0, 0.0, 0.02, 0.1] if mixed else [0.05], 0.0, mixed or cut == "min"),
                # (the middles of 2^24 equal parts: neither 0 nor 1)
                u=(torch.randint(0, 1 << 24, (n,), device="cuda", generator=g).double() + 0.5).mul(2.0 ** -24).float(),
                token=torch.empty(n, dtype=torch.int32, device="cuda"),
                logprob=torch.empty(n, dtype=torch.float32, device="cuda"),
                status=torch.zeros(1, dtype=torch.int32, device="cuda"))


# ------------------------------------------------------------------- one pass
def run(st):
    kind = st["case"]["kind"]
    if own:
        return {"append": _own_append, "attn": _own_attn, "sample": _own_sample}[kind](st)
    with torch.no_grad():
        return {"append": _plain_append, "attn": _plain_attn, "sample": _plain_sample}[kind](st)


def _appended(st):
    """What an append changes.  The pools are e4m3 numbers, and stand for that many of their block's scale."""
    out = dict(q=st["q_out"], k=st["k"], v=st["v"], scale=st["scale"])
    return out if st["summary"] is None else dict(out, summary=st["summary"])


def _own_append(st):
    import paper_2601_08670_gb300 as pced
    pced.kv_append(st["cache"], st["q"], st["nk"], st["nv"], rope=st["rope"],
                   tok_start=None if st["one"] else st["tok_start"], q_out=st["q_out"], status=st["status"])
    return _appended(st)


def _own_attn(st):
    import paper_2601_08670_gb300 as pced
    pced.paged_attention(st["cache"], st["q"], sel=st["sel"], out=st["out"], lse=st["lse"], ws=st["ws"])
    return dict(out=st["out"], lse=st["lse"])


def _own_sample(st):
    import paper_2601_08670_gb300 as pced
    pced.sample(st["x"], st["u"], temperature=st["temperature"], top_k=st["top_k"], top_p=st["top_p"],
                min_p=st["min_p"], token=st["token"], logprob=st["logprob"], status=st["status"])
    return dict(token=st["token"], logprob=st["logprob"])


def _rotated(x, rope):
    """Rotate-half of x [T, H, D] with the table's rows [T, D], in 32 bits and not rounded further."""
    D = x.shape[2]
    a, b, c, s = x[..., :D // 2].float(), x[..., D // 2:].float(), rope[:, None, :D // 2], rope[:, None, D // 2:]
    return torch.cat([a * c - b * s, b * c + a * s], dim=2)


def _plain_append(st):
    c, T = st["case"], st["T"]
    P, S = c["P"], c["S"]
    start, lens = st["tok_start"].long(), st["lens"].long()
    count = start[1:] - start[:-1]
    seq = torch.repeat_interleave(torch.arange(S, device="cuda"), count, output_size=T)
    row = lens[seq] - start[seq + 1] + torch.arange(T, device="cuda")
    q, k, v = st["q"], st["nk"].float(), st["nv"].float()
    if st["rope"] is not None:
        rope = st["rope"][row]
        q, k = _rotated(q, rope), _rotated(k, rope)
    st["q_out"].copy_(q)
    block, at = st["table"][seq, row // P].long(), row % P
    # the scales that the blocks' new rows need, [blocks, heads, 2]
    new = torch.stack([k, v], dim=2)  # [T, heads, 2, D]
    top = torch.where(torch.isfinite(new), new.abs(), 0.0).amax(dim=3)
    most = torch.zeros_like(st["scale"])
    most.scatter_reduce_(0, block[:, None, None].expand(top.shape), top, "amax")
    t_seq, t_block = st["touched"]
    first = (lens - count)[t_seq] - t_block * P  # of each touched block the first new row; the block starts anew from 0 on
    t_pool = st["table"][t_seq, t_block].long()
    before, need = st["scale"][t_pool], _steps(most[t_pool])
    scale = torch.where((first <= 0)[:, None, None], need, torch.maximum(before, need))
    st["scale"][t_pool] = scale
    # rows from before the call move where their block's scale grew
    ratio = before / scale
    held = (torch.arange(P, device="cuda") < first[:, None])[:, None, :, None]
    inverse = torch.ones_like(scale) / scale
    per_block = torch.zeros_like(st["scale"])
    per_block[t_pool] = inverse
    for i, pool in enumerate((st["k"], st["v"])):
        raw = pool.view(torch.uint8)
        mine = raw[t_pool]
        moved = (mine.view(E4M3).float() * ratio[:, :, i, None, None]).to(E4M3).view(torch.uint8)
        raw[t_pool] = torch.where(held & (ratio[:, :, i, None, None] != 1), moved, mine)
        raw[block, :, at] = (new[:, :, i] * per_block[block][:, :, i, None]).to(E4M3).view(torch.uint8)
    if st["summary"] is not None:  # a block whose row 0 is new starts anew
        summ = st["summary"].float()
        fresh = torch.zeros(summ.shape[0], dtype=torch.bool, device="cuda")
        fresh[block] = True
        fresh[t_pool] &= first <= 0
        summ[:, :, 0].masked_fill_(fresh[:, None, None], -127.0)
        summ[:, :, 1].masked_fill_(fresh[:, None, None], 127.0)
        x = k * (torch.ones_like(st["step"]) / st["step"])[:, None]
        where = block[:, None, None].expand(x.shape)
        summ[:, :, 0].scatter_reduce_(0, where, x.ceil().clamp_(-127, 127), "amax")
        summ[:, :, 1].scatter_reduce_(0, where, x.floor().clamp_(-127, 127), "amin")
        st["summary"].copy_(summ.to(torch.int8))
    return _appended(st)


def _plain_attn(st):
    c = st["case"]
    Hq, Hkv, D = HEADS[c["heads"]]
    S, P = c["S"], c["P"]
    table, n = st["table"].long(), st["lens"].long()
    if st["sel"] is None:
        logical = torch.arange(table.shape[1], device="cuda").expand(S, -1)
        blocks = table.clamp(min=0)
        head = slice(None)
        turn = (lambda x: x.transpose(1, 2))  # [S, Hkv, blocks, ...]
        logical = logical[:, None]
    else:
        logical = st["sel"].long()
        blocks = torch.gather(table[:, None].expand(-1, Hkv, -1), 2, logical.clamp(min=0))
        head = torch.arange(Hkv, device="cuda")[:, None]
        turn = (lambda x: x)
    k, v = (turn(x.view(torch.uint8)[blocks, head]).view(E4M3).float() *
            turn(st["scale"][blocks, head])[..., i, None, None] for i, x in enumerate((st["k"], st["v"])))
    row = logical[..., None] * P + torch.arange(P, device="cuda")
    live = ((logical[..., None] >= 0) & (row < n[:, None, None, None])).flatten(2)[:, :, None]  # [S, 1 or Hkv, 1, rows]
    q = st["q"].float().view(S, Hkv, -1, D)
    s = q @ k.flatten(2, 3).transpose(2, 3) * (1.0 / math.sqrt(D))
    s = s.masked_fill_(~live, -math.inf)
    top = s.amax(dim=3, keepdim=True)
    p = torch.exp(s - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(dim=3, keepdim=True)
    v = v.flatten(2, 3).masked_fill(~live.transpose(2, 3), 0.0)
    o = (p @ v) / torch.where(total == 0, 1.0, total)
    st["out"].copy_(o.reshape(S, Hq, D))
    st["lse"].copy_((top + total.log()).view(S, Hq))
    return dict(out=st["out"], lse=st["lse"])


def _plain_sample(st):
    # (64 bits: a sum of 150,000 weights in 32 misses the border of two tokens in one row of a few hundred)
    x = st["x"].double()
    n, V = x.shape
    t, p, low, u = (st[a].double()[:, None] for a in ("temperature", "top_p", "min_p", "u"))
    greedy = t == 0
    k = torch.where(greedy[:, 0] | (st["top_k"] == 1), 1, torch.where(st["top_k"] > 0, st["top_k"], V))[:, None]
    z = (x - x.amax(dim=1, keepdim=True)) / torch.where(greedy, 1.0, t)
    order = x.sort(dim=1, descending=True, stable=True).indices  # ties: the lowest token first
    at = torch.arange(V, device="cuda")
    w = z.exp()
    w_in_order = torch.where(at < k, w.gather(1, order), 0.0)
    before = w_in_order.cumsum(1) - w_in_order
    keep = (at < k) & (before < p * w_in_order.sum(1, keepdim=True)) & (w_in_order >= low) | (at == 0)
    w = torch.where(torch.zeros_like(keep).scatter_(1, order, keep), w, 0.0)
    sums = w.cumsum(1)
    total = sums[:, -1:]
    token = (sums <= u * total).sum(1, keepdim=True).clamp_(max=V - 1)
    st["token"].copy_(token[:, 0])
    logprob = z.gather(1, token) - total.log()
    st["logprob"].copy_(torch.where(k == 1, 0.0, logprob)[:, 0])
    return dict(token=st["token"], logprob=st["logprob"])


# ------------------------------------------------------------ what it has to do
def work(case):
    if case["kind"] == "sample":
        size = {"fp32": 4, "bf16": 2}[case["type"]]
        return {"bytes": case["rows"] * (case["V"] * size + 28), "flops": 3 * case["rows"] * case["V"]}
    Hq, Hkv, D = HEADS[case["heads"]]
    lens, S, P = _lengths(case), case["S"], case["P"]
    nb = (lens + P - 1) // P
    rows, blocks = int(lens.sum()), int(nb.sum())
    if case["kind"] == "append":
        T, touched = int(_new(case, lens).sum()), len(_touched(case, lens)[0])
        angles = 4 * D * min(T, int(lens.max())) if case["rope"] else 0
        summary = 2 * touched * Hkv * D if case["summary"] else 0
        return {"bytes": T * (4 * Hq + 6 * Hkv) * D + angles + touched * (8 * Hkv + 4) + summary + 8 * S,
                "flops": (3 * T * (Hq + Hkv) * D if case["rope"] else 0) + 4 * T * Hkv * D}
    if case["keep"]:
        rows = int(np.minimum(lens, case["keep"] * P - (nb * P - lens)).sum())
        blocks = int(np.minimum(nb, case["keep"]).sum())
    return {"bytes": rows * 2 * Hkv * D + blocks * (8 * Hkv + 4) + 6 * S * Hq * D + 4 * S * Hq + 4 * S,
            "flops": 4 * rows * Hq * D}


# --------------------------------------------------------- the same in 64 bits
def exact(case, seed):
    with torch.no_grad():
        st = prepare(case, seed)
        return {"append": _exact_append, "attn": _exact_attn, "sample": _exact_sample}[case["kind"]](case, st)


def _exact_append(c, st):
    lens, table = st["host"]
    m, P, D = _new(c, lens), c["P"], st["q"].shape[2]
    q, k, v = st["q"].double(), st["nk"].double(), st["nv"].double()
    if st["rope"] is not None:
        row = np.concatenate([np.arange(n - j, n) for n, j in zip(lens, m)])
        t = st["rope"].double()[_dev(row, torch.int64)][:, None]
        cos, sin = t[..., :D // 2], t[..., D // 2:]
        q, k = (torch.cat([x[..., :D // 2] * cos - x[..., D // 2:] * sin,
                           x[..., D // 2:] * cos + x[..., :D // 2] * sin], dim=2) for x in (q, k))
    scale = st["scale"].double().cpu().numpy()
    pools = [st["k"].double(), st["v"].double()]
    at = 0
    for s, (n, j) in enumerate(zip((int(x) for x in lens), (int(x) for x in m))):
        while j > 0:  # a block of the sequence at a time
            r0, b = (n - j) % P, int(table[s, (n - j) // P])
            here = min(j, P - r0)
            for i, x in enumerate((k, v)):
                x = x[at:at + here].transpose(0, 1)
                top = x.abs().amax(dim=(1, 2)).cpu().numpy()
                need = np.exp2(np.maximum(np.ceil(np.log2(np.maximum(top, 1e-300) / TOP)), LOWEST))
                now = need if r0 == 0 else np.maximum(scale[b, :, i], need)
                pools[i][b, :, :r0] *= _dev(scale[b, :, i] / now, torch.float64)[:, None, None]
                pools[i][b, :, r0:r0 + here] = x / _dev(now, torch.float64)[:, None, None]
                scale[b, :, i] = now
            j, at = j - here, at + here
    out = dict(q=q, k=pools[0], v=pools[1], scale=torch.from_numpy(scale))
    # (the summaries are counted from keys rounded to 32 bits: they have no value of their own in 64)
    return out if st["summary"] is None else dict(out, summary=None)


def _exact_attn(c, st):
    lens, table = st["host"]
    Hq, Hkv, D = HEADS[c["heads"]]
    P, G = c["P"], Hq // Hkv
    out = torch.zeros((c["S"], Hq, D), dtype=torch.float64, device="cuda")
    lse = torch.full((c["S"], Hq), -math.inf, dtype=torch.float64, device="cuda")
    pools = [x.view(torch.uint8) for x in (st["k"], st["v"])]
    for s, n in enumerate(int(x) for x in lens):
        nb = (n + P - 1) // P
        tab = _dev(table[s, :nb], torch.int64)
        for h in range(Hkv):
            heads = slice(h * G, (h + 1) * G)
            chosen = torch.arange(nb, device="cuda") if st["sel"] is None else st["sel"][s, h].long()
            chosen = chosen[chosen >= 0]
            row = (chosen[:, None] * P + torch.arange(P, device="cuda")).flatten()
            row = row[row < n]
            if not len(row):
                continue
            block = tab[row // P]
            k, v = (x[block, h, row % P].view(E4M3).double() * st["scale"][block, h, i].double()[:, None]
                    for i, x in enumerate(pools))
            z = st["q"][s, heads].double() @ k.T / math.sqrt(D)
            lse[s, heads] = torch.logsumexp(z, dim=1)
            out[s, heads] = torch.softmax(z, dim=1) @ v
    return dict(out=out, lse=lse)


def _exact_sample(c, st):
    x = st["x"].double().cpu().numpy()
    t, k, p, low, u = (st[a].double().cpu().numpy() for a in ("temperature", "top_k", "top_p", "min_p", "u"))
    token, logprob = np.zeros(c["rows"], np.int32), np.zeros(c["rows"])
    for i, z in enumerate(x):
        if t[i] == 0 or k[i] == 1:
            token[i] = z.argmax()
            continue
        z = (z - z.max()) / t[i]
        order = np.argsort(-z, kind="stable")[:int(k[i]) if k[i] > 0 else None]
        w = np.exp(z[order])
        sums = np.cumsum(w)
        if p[i] < 1:
            order = order[:1 + np.searchsorted(sums, p[i] * sums[-1])]
        order = order[:max(1, int((w[:len(order)] >= low[i]).sum()))]
        order = np.sort(order)
        sums = np.cumsum(np.exp(z[order]))
        token[i] = order[min(len(order) - 1, np.searchsorted(sums, u[i] * sums[-1], side="right"))]
        logprob[i] = z[token[i]] - np.log(sums[-1])
    return dict(token=torch.from_numpy(token), logprob=torch.from_numpy(logprob))
