"""The operators over paged caches together: the example's decode loop against the same loop in plain 64-bit PyTorch,
and pced_step's layer chain rebuilt from them."""
import math
import os
import subprocess
import sys

import pytest
import torch

import synth

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))


def make(blocks=0, steps=3, penalties=False, mask=None, seed=0):
    import paged_decode as ex
    B, N = 2, 2
    lens = [7, 150, 64, 20, 97, 33]
    model = ex.Model(L=2, Hq=8, Hkv=2, D=64, V=1000, rows=max(lens) + steps, seed=seed)
    g = torch.Generator(device="cuda").manual_seed(seed + 5)
    r = torch.rand((B, N), device="cuda", generator=g)
    pen = torch.tensor([[1.3, 0.5, 0.25]] * B, device="cuda") if penalties else None
    loop = ex.Loop(model, B, N, lens, steps, torch.full((B, N), 0.5, device="cuda"), r, blocks=blocks, penalties=pen,
                   mask=mask)
    hidden = torch.randn((sum(lens), model.Hq * model.D), device="cuda", generator=g)
    loop.load_documents(hidden)
    return loop, hidden, lens


def plain_hidden(loop, hidden, lens, tokens):
    """Final hidden states of the last step, all arithmetic in 64 bits, for the given tokens (one list per query)."""
    m = loop.model
    w = [(a.double(), b.double()) for a, b in zip(m.qkv, m.out)]

    def norm(x):
        return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)

    def rot(x, pos):
        t = m.rope.double()[pos][:, None]
        a, b, co, si = x[..., :32], x[..., 32:], t[..., :32], t[..., 32:]
        return torch.cat([a * co - b * si, b * co + a * si], -1)

    out, at = [], 0
    for s, n in enumerate(lens):
        doc = hidden[at:at + n].double()
        at += n
        kv = []
        for wq, _ in w:
            y = (norm(doc) @ wq.T).view(n, -1, 64)
            kv.append((rot(y[:, 8:10], torch.arange(n, device="cuda")), y[:, 10:]))
        for i, tok in enumerate([0] + tokens[s // 3][:-1]):
            x = m.embed[tok].double()[None]
            for layer, (wq, wo) in enumerate(w):
                y = (norm(x) @ wq.T).view(1, -1, 64)
                pos = torch.tensor([n + i], device="cuda")
                k = torch.cat([kv[layer][0], rot(y[:, 8:10], pos)])
                v = torch.cat([kv[layer][1], y[:, 10:]])
                kv[layer] = (k, v)
                q = rot(y[:, :8], pos).view(2, 4, 64)
                p = torch.softmax(torch.einsum("hgd,nhd->hgn", q, k) / 8.0, -1)
                x = x + torch.einsum("hgn,nhd->hgd", p, v).reshape(1, -1) @ wo.T
        out.append(norm(x)[0])
    return torch.stack(out)


def test_loop_matches_the_plain_one(cuda_ok):
    loop, hidden, lens = make(steps=3)
    for _ in range(3):
        loop.step()
    assert loop.device_status() == 0
    want = plain_hidden(loop, hidden, lens, loop.history.tolist())
    # each layer rounds its inputs, projections, queries, keys and output to bf16 (2^-9 each, about six of them), and
    # two layers add up: 12 * 2^-9 of the rows' unit size, in the mean over a row
    err = (loop.hidden.double() - want).square().mean(1).sqrt()
    assert float(err.max()) <= 12 * 2.0 ** -9


def test_all_blocks_selected_is_the_dense_loop(cuda_ok):
    dense, hidden, _ = make(blocks=0)
    every, _, _ = make(blocks=64)
    few, _, _ = make(blocks=3)
    for _ in range(3):
        for loop in (dense, every, few):
            loop.step()
    assert dense.device_status() == every.device_status() == few.device_status() == 0
    assert torch.equal(dense.history, every.history) and torch.equal(dense.hidden, every.hidden)
    assert not torch.equal(dense.hidden, few.hidden)


def test_penalties_and_masks_steer_the_choice(cuda_ok):
    mask = torch.zeros((2, 32), dtype=torch.int32, device="cuda")
    mask[:, 3] = 0b1010000  # tokens 100 and 102
    loop, _, _ = make(steps=3, penalties=True, mask=mask)
    free, _, _ = make(steps=3, mask=mask)
    for _ in range(3):
        loop.step()
        free.step()
    assert set(loop.history.flatten().tolist()) <= {100, 102}
    assert set(free.history.flatten().tolist()) <= {100, 102}
    lp = loop.logprobs
    assert bool(torch.isneginf(lp[:, :100]).all()) and bool(torch.isfinite(lp[:, 100]).all())


def test_the_example_runs(cuda_ok):
    res = subprocess.run([sys.executable, os.path.join(ROOT, "examples", "paged_decode.py"), "--steps", "4"],
                         capture_output=True, text=True, timeout=300)
    assert res.returncode == 0, res.stderr[-2000:]
    assert res.stdout.count("tokens") == 2


def test_operators_rebuild_the_step(cuda_ok):
    # pced_step's weight-free chain over its own paged pool, from the operators
    import paper_2601_08670_gb300 as pced
    w = synth.get("tiny")
    P = 64
    t = synth.device_inputs(w, "cuda", paged=P)
    lay = t["paged_layout"]
    dm = pced.dims(w.B, w.N, w.L, w.Hq, w.Hkv, w.D, w.V)
    pools = [t[x].clone().view(w.L, lay.num_blocks, w.Hkv, P, w.D) for x in ("k_cache", "v_cache")]
    lens = t["seq_len"].clone()
    caches = [pced.PagedCache(pools[0][l], pools[1][l], t["block_table"], lens) for l in range(w.L)]
    dec = pced.decoder_from_inputs(dm, t, gamma=w.gamma, max_steps=w.steps, bos=w.bos, keep_hidden=True)
    tok = torch.full((w.B,), w.bos, dtype=torch.long, device="cuda")
    for step in range(3):
        dec.step()
        lens += 1
        x = t["embed"][tok].float().repeat_interleave(w.N + 1, 0)
        for cache in caches:
            u = (x * torch.rsqrt(x.square().mean(1, keepdim=True) + 1e-6)).bfloat16().view(w.S, w.Hq, w.D)
            q = pced.kv_append(cache, u, u[:, :w.Hkv], u[:, w.Hkv:2 * w.Hkv])
            x = x + pced.paged_attention(cache, q).view(w.S, -1)
        h = (x * torch.rsqrt(x.square().mean(1, keepdim=True) + 1e-6)).bfloat16()
        # bf16 roundings may turn where fp32 sums run in another order: almost all of the states are equal
        assert float((h == dec.hidden).float().mean()) >= 0.98
        lp, _ = pced.lm_head_logprobs(h, t["w_unembed"])
        token, expert, _ = pced.contrastive_select(lp, t["beta"], t["r"], w.gamma)
        gaps = dec.gap_trace[:, step]
        for b in range(w.B):
            if float(gaps[b].min()) >= 1e-3:
                assert int(token[b]) == int(dec.history[b, step]) and int(expert[b]) == int(dec.expert_trace[b, step])
        tok = dec.history[:, step].long()
    assert dec.status() == 0


def test_operators_in_one_graph(cuda_ok):
    # a layer's calls and the logits' captured together: replays follow the lengths and buffers on the device
    import numpy as np
    import paged_ref as ref
    import paper_2601_08670_gb300 as pced
    rng = np.random.default_rng(31)
    Hq, Hkv, D, P, lens = 8, 2, 64, 16, [100, 700, 0, 33]
    c = ref.make_cache(rng, lens, Hkv, D, P, spare=8, spoil=False)
    S = len(lens)
    cache = ref.to_device(c, np.zeros((len(c["k"]), Hkv, 2, D), np.int8))
    pced.block_summaries(cache)
    base = {n: getattr(cache, n).clone() for n in ("k", "v", "summary", "seq_len")}
    qkv = torch.empty((S, Hq + 2 * Hkv, D), dtype=torch.bfloat16, device="cuda")
    rope = pced.rope_table(1e4, D, 1000)
    bufs = dict(q=torch.empty((S, Hq, D), dtype=torch.bfloat16, device="cuda"),
                sel=torch.empty((S, Hkv, 6), dtype=torch.int32, device="cuda"),
                out=torch.empty((S, Hq, D), device="cuda"), y=torch.empty((S, 500), device="cuda"))
    ws = pced.workspace(pced.paged_attention_workspace_size(S, Hq, Hkv, D), "cuda")
    x = torch.from_numpy(rng.normal(size=(S, 500)).astype(np.float32)).cuda()
    hist, n_hist = torch.zeros((2, 4), dtype=torch.int32, device="cuda"), torch.full((2,), 4, dtype=torch.int32,
                                                                                    device="cuda")
    pen = torch.full((2, 3), 1.5, device="cuda")
    one = (cache.seq_len > 0).to(torch.int32)

    def layer():
        cache.seq_len.add_(one)
        pced.kv_append(cache, qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:], rope=rope, q_out=bufs["q"])
        pced.block_select(cache, bufs["q"], 6, sel=bufs["sel"])
        pced.paged_attention(cache, bufs["q"], sel=bufs["sel"], out=bufs["out"], ws=ws)
        pced.logits_process(x, 2, history=hist, history_len=n_hist, penalties=pen, out=bufs["y"])

    inputs = [ref.rng_bf16(rng, (S, Hq + 2 * Hkv, D)).cuda() for _ in range(3)]
    results = []
    for graphed in (False, True):
        for n, t in base.items():
            getattr(cache, n).copy_(t)
        if graphed:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                layer()
        got = []
        for v in inputs:
            qkv.copy_(v)
            g.replay() if graphed else layer()
            got.append([t.clone() for t in (*bufs.values(), cache.k, cache.summary)])
        results.append(got)
    torch.cuda.synchronize()
    assert pced.device_status(ws) == 0
    for a, b in zip(*results):
        assert all(torch.equal(s, t) for s, t in zip(a, b))
