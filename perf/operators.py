"""Measured work of the operators that a program with its own layers decodes with over paged caches.

Five operators, each with its plain form beside the library's call:

* ``append``   ``kv_append``: new keys and values into the pages, rotated on the way, queries rotated beside them,
  and the pages' key summaries brought up to date;
* ``summary``  ``block_summaries``: the summaries of caches that were built elsewhere (documents encoded offline);
* ``select``   ``block_select``: the blocks that each query's sequences attend to, by a score of the summaries;
* ``attn``     ``paged_attention``: one new token per sequence, over all blocks or over the selected ones;
* ``logits``   ``logits_process``: penalties for repeated tokens, biases and grammar masks.

Shapes are those of the synthetic workloads and of the tests; the inputs are generated here, from the seed alone.
"""
import math

import numpy as np
import torch

own = False  # True: `run` makes the library's calls; False: the plain forms

ROOM = 64    # rows kept free in every cache for the tokens to come
QUERY = 32   # rows of the question, which every cache holds after its document
FORCED = 1 << 30

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
        dict(name="append_step", kind="append", heads="32/8/128", S=9, lo=2081, hi=2081, new=1, P=64, idle=0, rope=True),
        # sixteen ragged documents of about 1024 rows encoded in one pass: the largest append
        dict(name="append_docs", kind="append", heads="32/8/128", S=16, lo=256, hi=2048, new=0, P=64, idle=0, rope=True),
        # summaries of one query's eight documents and amateur
        dict(name="summary_docs", kind="summary", heads="32/8/128", S=9, lo=2080, hi=2080, P=64, idle=0),
        # ... of sixteen queries' ragged documents
        dict(name="summary_batch", kind="summary", heads="32/8/128", S=272, lo=256, hi=2048, P=128, idle=0),
        # choosing among the blocks of documents of 8192 rows
        dict(name="select_docs", kind="select", heads="32/8/128", S=9, lo=8224, hi=8224, P=64, idle=0, keep=32),
        # ... of 32 very long ones
        dict(name="select_long", kind="select", heads="32/8/128", S=33, lo=65568, hi=131104, P=64, idle=0, keep=64),
        # the tiny workload's layer: the smallest attention, where launches count
        dict(name="attn_tiny", kind="attn", heads="8/2/64", S=3, lo=257, hi=257, P=64, idle=0, keep=0),
        # one layer over eight documents of 2048 rows, all blocks
        dict(name="attn_docs", kind="attn", heads="32/8/128", S=9, lo=2081, hi=2081, P=64, idle=0, keep=0),
        # sixteen queries' ragged documents at once: the largest layer
        dict(name="attn_batch", kind="attn", heads="32/8/128", S=272, lo=256, hi=2048, P=128, idle=0, keep=0),
        # 64 selected blocks of every document of 16384 rows, seven query heads per kv head
        dict(name="attn_select", kind="attn", heads="28/4/128", S=17, lo=16416, hi=16416, P=64, idle=0, keep=64),
        # one query's experts before the choice of a token: a short history, a grammar's mask
        dict(name="logits_docs", kind="logits", B=1, R=9, V=128256, hist=64, bias=16, mask=True),
        # sixteen queries' experts, their prompts among the tokens that count as repeated
        dict(name="logits_batch", kind="logits", B=16, R=17, V=151936, hist=4096, bias=300, mask=True),
    ]


def _log(rng, lo, hi):
    """A whole number spread over the logarithm of [lo, hi]."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["append", "summary", "select", "attn", "attn", "attn", "logits"])
    if kind == "logits":
        B = rng.choice([1, 1, 2, 3, 5, 8, 16])
        return dict(kind=kind, B=B, R=_log(rng, 2, min(64, 272 // B)), V=_log(rng, 1000, 151936),
                    hist=_log(rng, 1, 8192), bias=rng.choice([0, 1, 16, 300]), mask=rng.random() < 0.6)
    heads = rng.choice(sorted(HEADS))
    Hq, Hkv, D = HEADS[heads]
    S = _log(rng, 1, 272)
    P = rng.choice([16, 32, 64, 64, 128, 192, 256])
    # rows of a sequence: at most about what the largest listed case of the kind holds
    most = {"append": 18_000, "summary": 300_000, "select": 3_000_000 * P // 64, "attn": 300_000}[kind]
    hi = _log(rng, 16, max(32, min(131_072, most // S)))
    lo = rng.choice([hi, max(1, hi // rng.randint(2, 16))])
    c = dict(kind=kind, heads=heads, S=S, lo=lo, hi=hi, P=P, idle=rng.choice([0, 0, 1]) if S > 1 else 0)
    if kind == "append":
        c.update(new=rng.choice([0, 1, 1, 2, QUERY, 100]), rope=rng.random() < 0.8)
    if kind == "select":
        c["keep"] = _log(rng, 2, 256)
    if kind == "attn":
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
    table = np.full((len(lens), int(nblk.max())), -1, np.int64)
    at = 0
    for s, n in enumerate(nblk):
        table[s, :n] = order[at:at + n]
        at += n
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


def prepare(case, seed):
    if case["kind"] == "logits":
        return _prepare_logits(case, seed)
    Hq, Hkv, D = HEADS[case["heads"]]
    S, P = case["S"], case["P"]
    lens, g = _lengths(case), _gen(seed)
    table, nblocks = _pages(lens, P, seed)
    st = dict(case=case, lens=_dev(lens, torch.int32), table=_dev(table, torch.int32), host=(lens, table, nblocks),
              status=torch.zeros(1, dtype=torch.int32, device="cuda"), k=None, v=None, summary=None, step=None)
    if case["kind"] != "select":  # a choice reads the summaries alone
        st["k"] = _normal((nblocks, Hkv, P, D), 1.0, g)
        live = _dev(_live(lens, table, nblocks, P), torch.int64)
    if case["kind"] in ("append", "attn"):
        st["v"] = _normal((nblocks, Hkv, P, D), 1.0, g)
    if case["kind"] != "attn":
        st["step"] = torch.full((Hkv,), 5.0 / 127.0, device="cuda") * (1 + 0.25 * torch.rand(
            Hkv, device="cuda", generator=g))
    if case["kind"] == "append":
        m = _new(case, lens)
        T = int(m.sum())
        qkv = _normal((T, Hq + 2 * Hkv, D), 1.0, g)  # one projection's output
        st.update(q=qkv[:, :Hq], nk=qkv[:, Hq:Hq + Hkv], nv=qkv[:, Hq + Hkv:], T=T,
                  q_out=torch.empty((T, Hq, D), dtype=torch.bfloat16, device="cuda"),
                  tok_start=_dev(np.concatenate([[0], np.cumsum(m)]), torch.int32),
                  one=case["new"] == 1 and case["idle"] == 0,
                  rope=_rope_table(max(1, int(lens.max())), D) if case["rope"] else None)
        spread = torch.randint(60, 100, (nblocks, Hkv, 2, D), device="cuda", generator=g, dtype=torch.int32)
        spread[:, :, 1] *= -1
        st["summary"] = spread.to(torch.int8)
    elif case["kind"] == "summary":
        _spoil(st["k"], live)
        st["summary"] = torch.zeros((nblocks, Hkv, 2, D), dtype=torch.int8, device="cuda")
    elif case["kind"] == "select":
        st["q"] = _normal((S, Hq, D), 1.0, g)
        # blocks differ by their mean; its largest and smallest row lie about 2.4 away
        mid = _normal((nblocks, Hkv, 1, D), 18.0, g, torch.float32)
        side = _normal((nblocks, Hkv, 2, D), 6.0, g, torch.float32).abs_() + 48.0
        side[:, :, 1] *= -1
        st["summary"] = side.add_(mid).round_().clamp_(-127, 127).to(torch.int8)
        st["sel"] = torch.empty((S, Hkv, case["keep"]), dtype=torch.int32, device="cuda")
    else:
        _spoil(st["k"], live)
        _spoil(st["v"], live)
        st.update(q=_normal((S, Hq, D), 1.0, g), sel=_choice(case, lens, g) if case["keep"] else None,
                  out=torch.empty((S, Hq, D), dtype=torch.float32, device="cuda"),
                  lse=torch.empty((S, Hq), dtype=torch.float32, device="cuda"))
    if own:
        import paper_2601_08670_gb300 as pced
        st["cache"] = pced.PagedCache(st["k"], st["v"], st["table"], st["lens"], block_rows=P, summary=st["summary"],
                                      key_step=st["step"])
        if case["kind"] == "attn":
            st["ws"] = pced.workspace(pced.paged_attention_workspace_size(S, Hq, Hkv, D), "cuda")
    return st


def _spoil(pool, live):
    """What no sequence has written yet is not a number."""
    P = pool.shape[2]
    dead = torch.arange(P, device="cuda")[None] >= live[:, None]
    pool.masked_fill_(dead[:, None, :, None], float("nan"))


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


def _prepare_logits(c, seed):
    B, R, V, n = c["B"], c["R"], c["V"], c["hist"]
    g = _gen(seed)
    x = _normal((B * R, V), 2.5, g, torch.float32)
    # tokens repeat: low numbers far more often than high ones
    hist = (torch.rand((B, n), device="cuda", generator=g) ** 4 * V).to(torch.int32).clamp_(0, V - 1)
    hlen = torch.randint(n // 2, n + 1, (B,), device="cuda", generator=g, dtype=torch.int32)
    pen = torch.rand((B, 3), device="cuda", generator=g)  # repetition, frequency, presence
    pen[:, 0] += 1.0
    st = dict(case=c, x=x, hist=hist, hlen=hlen, pen=pen, ids=None, bias=None, mask=None, mask_row=None,
              out=torch.empty_like(x), status=torch.zeros(1, dtype=torch.int32, device="cuda"))
    if c["bias"]:
        at = np.stack([np.random.default_rng([seed, b]).permutation(V)[:c["bias"]] for b in range(B)])
        st.update(ids=_dev(at, torch.int32), bias=_normal((B, c["bias"]), 3.0, g, torch.float32))
    if c["mask"]:  # five states of a grammar, some queries outside of one
        st.update(mask=torch.randint(-2 ** 31, 2 ** 31, (5, (V + 31) // 32), device="cuda", generator=g,
                                     dtype=torch.int64).to(torch.int32),
                  mask_row=torch.randint(-1, 5, (B,), device="cuda", generator=g, dtype=torch.int32))
    return st


# ------------------------------------------------------------------- one pass
def run(st):
    kind = st["case"]["kind"]
    if own:
        return {"append": _own_append, "summary": _own_summary, "select": _own_select, "attn": _own_attn,
                "logits": _own_logits}[kind](st)
    with torch.no_grad():
        return {"append": _plain_append, "summary": _plain_summary, "select": _plain_select, "attn": _plain_attn,
                "logits": _plain_logits}[kind](st)


def _own_append(st):
    import paper_2601_08670_gb300 as pced
    pced.kv_append(st["cache"], st["q"], st["nk"], st["nv"], rope=st["rope"],
                   tok_start=None if st["one"] else st["tok_start"], q_out=st["q_out"], status=st["status"])
    return dict(q=st["q_out"], k=st["k"], v=st["v"], summary=st["summary"])


def _own_summary(st):
    import paper_2601_08670_gb300 as pced
    return pced.block_summaries(st["cache"], status=st["status"])


def _own_select(st):
    import paper_2601_08670_gb300 as pced
    return pced.block_select(st["cache"], st["q"], st["case"]["keep"], n_first=1, n_last=1, sel=st["sel"],
                             status=st["status"])


def _own_attn(st):
    import paper_2601_08670_gb300 as pced
    pced.paged_attention(st["cache"], st["q"], sel=st["sel"], out=st["out"], lse=st["lse"], ws=st["ws"])
    return dict(out=st["out"], lse=st["lse"])


def _own_logits(st):
    import paper_2601_08670_gb300 as pced
    return pced.logits_process(st["x"], st["case"]["R"], history=st["hist"], history_len=st["hlen"],
                               penalties=st["pen"], bias_ids=st["ids"], bias=st["bias"], mask=st["mask"],
                               mask_row=st["mask_row"], out=st["out"], status=st["status"])


def _rotated(x, rope):
    """Rotate-half of x [T, H, D] with the table's rows [T, D], in 32 bits."""
    D = x.shape[2]
    a, b, c, s = x[..., :D // 2].float(), x[..., D // 2:].float(), rope[:, None, :D // 2], rope[:, None, D // 2:]
    return torch.cat([a * c - b * s, b * c + a * s], dim=2).to(x.dtype)


def _inverse(step):
    return torch.ones_like(step) / step


def _plain_append(st):
    c, T = st["case"], st["T"]
    P, S = c["P"], c["S"]
    start = st["tok_start"].long()
    seq = torch.repeat_interleave(torch.arange(S, device="cuda"), start[1:] - start[:-1], output_size=T)
    row = st["lens"].long()[seq] - start[seq + 1] + torch.arange(T, device="cuda")
    q, k = st["q"], st["nk"]
    if st["rope"] is not None:
        rope = st["rope"][row]
        q, k = _rotated(q, rope), _rotated(k, rope)
    st["q_out"].copy_(q)
    block, at = st["table"][seq, row // P].long(), row % P
    st["k"][block, :, at] = k
    st["v"][block, :, at] = st["nv"]
    # summaries: a block whose row 0 is new starts anew
    summ = st["summary"].float()
    fresh = torch.zeros(summ.shape[0], dtype=torch.bool, device="cuda")
    fresh[block[at == 0]] = True
    summ[:, :, 0].masked_fill_(fresh[:, None, None], -127.0)
    summ[:, :, 1].masked_fill_(fresh[:, None, None], 127.0)
    x = k.float() * _inverse(st["step"])[:, None]
    where = block[:, None, None].expand(x.shape)
    summ[:, :, 0].scatter_reduce_(0, where, x.ceil().clamp_(-127, 127), "amax")
    summ[:, :, 1].scatter_reduce_(0, where, x.floor().clamp_(-127, 127), "amin")
    st["summary"].copy_(summ.to(torch.int8))
    return dict(q=st["q_out"], k=st["k"], v=st["v"], summary=st["summary"])


def _plain_summary(st):
    P, nblocks = st["case"]["P"], st["summary"].shape[0]
    table = st["table"].long()
    rows = (st["lens"].long()[:, None] - torch.arange(table.shape[1], device="cuda") * P).clamp(0, P)
    live = torch.zeros(nblocks + 1, dtype=torch.long, device="cuda")  # the last entry takes the table's empty places
    live[torch.where(table < 0, nblocks, table)] = rows
    live = live[:-1, None, None, None]
    x = st["k"].float() * _inverse(st["step"])[:, None, None]
    dead = torch.arange(P, device="cuda")[:, None] >= live
    mx = x.ceil().clamp_(-127, 127).masked_fill_(dead, -127.0).amax(dim=2)
    mn = x.floor().clamp_(-127, 127).masked_fill_(dead, 127.0).amin(dim=2)
    new = torch.stack([mx, mn], dim=2).to(torch.int8)
    st["summary"].copy_(torch.where(live > 0, new, st["summary"]))
    return st["summary"]


def _plain_select(st):
    c = st["case"]
    Hq, Hkv, D = HEADS[c["heads"]]
    S, P, keep = c["S"], c["P"], c["keep"]
    # the group's pooled query, in steps of a 127th of its largest part
    q = st["q"].float().view(S, Hkv, -1, D)
    pos, neg = q[:, :, 0].clamp(min=0), q[:, :, 0].clamp(max=0)
    for i in range(1, Hq // Hkv):
        pos, neg = pos + q[:, :, i].clamp(min=0), neg + q[:, :, i].clamp(max=0)
    pooled = torch.stack([pos, neg], dim=2)
    top = pooled.abs().amax(dim=(2, 3), keepdim=True)
    scale = torch.where(top > 0, torch.full_like(top, 127.0) / top, 0.0)
    pooled = (pooled * scale).round()
    # whole numbers below 2^24, so that sums in 32 bits are exact
    summ = st["summary"][st["table"].clamp(min=0).long()].float()  # [S, blocks, Hkv, 2, D]
    score = (summ * pooled[:, None]).sum(dim=(3, 4)).long().transpose(1, 2)
    nb = ((st["lens"].long() + P - 1) // P)[:, None, None]
    j = torch.arange(score.shape[2], device="cuda")
    score = torch.where((j < 1) | (j >= nb - 1), FORCED, score)
    key = torch.where(j < nb, (score << 20) - j, torch.iinfo(torch.int64).min)
    idx = key.topk(min(keep, key.shape[2]), dim=2).indices
    idx = torch.where(idx < nb, idx, key.shape[2]).sort(dim=2).values
    st["sel"].fill_(-1)
    st["sel"][:, :, :idx.shape[2]] = torch.where(idx == key.shape[2], -1, idx)
    return st["sel"]


def _plain_attn(st):
    c = st["case"]
    Hq, Hkv, D = HEADS[c["heads"]]
    S, P = c["S"], c["P"]
    table, n = st["table"].long(), st["lens"].long()
    if st["sel"] is None:
        logical = torch.arange(table.shape[1], device="cuda").expand(S, -1)
        blocks = table.clamp(min=0)
        k, v = (x[blocks].transpose(1, 2) for x in (st["k"], st["v"]))  # [S, Hkv, blocks, P, D]
        logical = logical[:, None]
    else:
        logical = st["sel"].long()
        blocks = torch.gather(table[:, None].expand(-1, Hkv, -1), 2, logical.clamp(min=0))
        head = torch.arange(Hkv, device="cuda")[:, None]
        k, v = (x[blocks, head] for x in (st["k"], st["v"]))
    row = logical[..., None] * P + torch.arange(P, device="cuda")
    live = ((logical[..., None] >= 0) & (row < n[:, None, None, None])).flatten(2)[:, :, None]  # [S, 1 or Hkv, 1, rows]
    q = st["q"].float().view(S, Hkv, -1, D)
    s = q @ k.float().flatten(2, 3).transpose(2, 3) * (1.0 / math.sqrt(D))
    s = s.masked_fill_(~live, -math.inf)
    top = s.amax(dim=3, keepdim=True)
    p = torch.exp(s - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(dim=3, keepdim=True)
    v = v.float().flatten(2, 3).masked_fill(~live.transpose(2, 3), 0.0)
    o = (p @ v) / torch.where(total == 0, 1.0, total)
    st["out"].copy_(o.reshape(S, Hq, D))
    st["lse"].copy_((top + total.log()).view(S, Hq))
    return dict(out=st["out"], lse=st["lse"])


def _plain_logits(st):
    c = st["case"]
    B, R, V, n = c["B"], c["R"], c["V"], c["hist"]
    x = st["x"].view(B, R, V)
    seen = torch.arange(n, device="cuda") < st["hlen"][:, None]
    count = torch.zeros((B, V + 1), device="cuda")  # the last entry takes what does not count
    count.scatter_add_(1, torch.where(seen, st["hist"].long(), V), torch.ones((B, n), device="cuda"))
    count = count[:, None, :V]
    rep, freq, pres = st["pen"].view(B, 3, 1, 1).unbind(1)
    y = torch.where(x > 0, x / rep, x * rep) - (count * freq + pres)
    y = torch.where(count > 0, y, x)
    if st["ids"] is not None:
        add = torch.zeros((B, V), device="cuda").scatter_(1, st["ids"].long(), st["bias"])
        y = y + add[:, None]
    if st["mask"] is not None:
        bits = st["mask"][st["mask_row"].long().clamp(min=0)]
        v = torch.arange(V, device="cuda")
        allowed = ((bits[:, v >> 5] >> (v & 31)) & 1 != 0) | (st["mask_row"] < 0)[:, None]
        y = torch.where(allowed[:, None], y, -math.inf)
    st["out"].copy_(y.view(B * R, V))
    return st["out"]


# ------------------------------------------------------------ what it has to do
def work(case):
    if case["kind"] == "logits":
        B, R, V = case["B"], case["R"], case["V"]
        words = 4 * min(5, B) * ((V + 31) // 32) if case["mask"] else 0
        return {"bytes": 8 * B * R * V + B * (4 * case["hist"] + 8 * case["bias"] + 20) + words, "flops": 4 * B * R * V}
    Hq, Hkv, D = HEADS[case["heads"]]
    lens, S, P = _lengths(case), case["S"], case["P"]
    nb = (lens + P - 1) // P
    rows, blocks = int(lens.sum()), int(nb.sum())
    if case["kind"] == "append":
        m = _new(case, lens)
        T, touched = int(m.sum()), int((nb - (lens - m) // P).sum())
        table = 4 * D * min(T, int(lens.max())) if case["rope"] else 0
        return {"bytes": 4 * T * (Hq + 2 * Hkv) * D + table + 2 * touched * Hkv * D + 8 * S + 4 * touched,
                "flops": (3 * T * (Hq + Hkv) * D if case["rope"] else 0) + 5 * T * Hkv * D}
    if case["kind"] == "summary":
        return {"bytes": rows * 2 * Hkv * D + blocks * (2 * Hkv * D + 4) + 4 * S, "flops": 5 * rows * Hkv * D}
    if case["kind"] == "select":
        return {"bytes": blocks * (2 * Hkv * D + 4) + 2 * S * Hq * D + 4 * S * Hkv * case["keep"] + 4 * S,
                "flops": 4 * blocks * Hkv * D}
    if case["keep"]:
        rows = int(np.minimum(lens, case["keep"] * P - (nb * P - lens)).sum())
    return {"bytes": rows * 4 * Hkv * D + 6 * S * Hq * D + 4 * S * Hq + 4 * S, "flops": 4 * rows * Hq * D}


# --------------------------------------------------------- the same in 64 bits
def exact(case, seed):
    with torch.no_grad():
        st = prepare(case, seed)
        return {"append": _exact_append, "summary": _exact_summary, "select": _exact_select, "attn": _exact_attn,
                "logits": _exact_logits}[case["kind"]](case, st)


def _exact_append(c, st):
    lens, table, _ = st["host"]
    m, P, D = _new(c, lens), c["P"], st["q"].shape[2]
    row = np.concatenate([np.arange(n - k, n) for n, k in zip(lens, m)])
    seq = np.repeat(np.arange(len(lens)), m)
    q, k = st["q"].double(), st["nk"].double()
    if st["rope"] is not None:
        t = st["rope"].double()[_dev(row, torch.int64)][:, None]
        cos, sin = t[..., :D // 2], t[..., D // 2:]
        q, k = (torch.cat([x[..., :D // 2] * cos - x[..., D // 2:] * sin,
                           x[..., D // 2:] * cos + x[..., :D // 2] * sin], dim=2) for x in (q, k))
    pools = [st["k"].double(), st["v"].double()]
    block, at = _dev(table[seq, row // P], torch.int64), _dev(row % P, torch.int64)
    for pool, x in zip(pools, (k, st["nv"].double())):
        pool[block, :, at] = x
    # the summaries are counted from the rounded keys: they have no value of their own in 64 bits
    return dict(q=q, k=pools[0], v=pools[1], summary=None)


def _exact_summary(c, st):
    lens, table, _ = st["host"]
    P, out = c["P"], st["summary"].clone()
    inv = _dev(np.float32(1.0) / st["step"].cpu().numpy(), torch.float64)[:, None]
    for s, n in enumerate(lens):
        for j in range((int(n) + P - 1) // P):
            b = int(table[s, j])
            # (the product of a bf16 and an fp32 number is whole in 64 bits; its rounding to fp32 is the definition's)
            x = (st["k"][b, :, :int(n) - j * P].double() * inv[:, None]).float()
            out[b, :, 0] = x.amax(1).ceil().clamp(-127, 127)
            out[b, :, 1] = x.amin(1).floor().clamp(-127, 127)
    return out


def _exact_select(c, st):
    lens, table, _ = st["host"]
    Hq, Hkv, D = HEADS[c["heads"]]
    q = st["q"].float().cpu().numpy().reshape(c["S"], Hkv, Hq // Hkv, D)
    summ = st["summary"].view(-1, Hkv, 2 * D).cpu().numpy()
    out = np.full((c["S"], Hkv, c["keep"]), -1, np.int32)
    for s, n in enumerate(lens):
        nb = (int(n) + c["P"] - 1) // c["P"]
        if not nb:
            continue
        of_s = summ[table[s, :nb]]
        for h in range(Hkv):
            parts = np.zeros((2, D), np.float32)
            for x in q[s, h]:
                parts += np.stack([np.maximum(x, 0), np.minimum(x, 0)])
            steps = np.rint(parts * (np.float32(127) / np.abs(parts).max())).reshape(-1).astype(np.float64)
            score = of_s[:, h].astype(np.float64) @ steps
            score[0] = score[-1] = FORCED
            best = np.lexsort((np.arange(nb), -score))[:c["keep"]]
            out[s, h, :len(best)] = np.sort(best)
    return torch.from_numpy(out)


def _exact_attn(c, st):
    lens, table, _ = st["host"]
    Hq, Hkv, D = HEADS[c["heads"]]
    P, G = c["P"], Hq // Hkv
    out = torch.zeros((c["S"], Hq, D), dtype=torch.float64, device="cuda")
    lse = torch.full((c["S"], Hq), -math.inf, dtype=torch.float64, device="cuda")
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
            k, v = (x[tab[row // P], h, row % P].double() for x in (st["k"], st["v"]))
            z = st["q"][s, heads].double() @ k.T / math.sqrt(D)
            lse[s, heads] = torch.logsumexp(z, dim=1)
            out[s, heads] = torch.softmax(z, dim=1) @ v
    return dict(out=out, lse=lse)


def _exact_logits(c, st):
    B, R, V = c["B"], c["R"], c["V"]
    y = st["x"].double().view(B, R, V)
    for b in range(B):
        tok, times = torch.unique(st["hist"][b, :int(st["hlen"][b])].long(), return_counts=True)
        rep, freq, pres = st["pen"][b].double()
        x = y[b][:, tok]
        y[b][:, tok] = torch.where(x > 0, x / rep, x * rep) - times * freq - pres
        if st["ids"] is not None:
            y[b].index_add_(1, st["ids"][b].long(), st["bias"][b].double().expand(R, -1))
        if st["mask"] is not None and int(st["mask_row"][b]) >= 0:
            words = st["mask"][int(st["mask_row"][b])].cpu().numpy().astype("<i4")
            bits = np.unpackbits(words.view(np.uint8), bitorder="little")[:V]
            y[b][:, _dev(bits == 0, torch.bool)] = -math.inf
    return y.view(B * R, V)
