"""The operators over 8-bit caches and sample together, as a decode loop calls them: against their definitions in 64 bits,
captured as one graph, on two streams at once, in the example and in the bounds-checked build."""
import json
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import cache8_ref as ref8
import decode8_checked_run
import paged_ref as ref
import sample_ref

pytestmark = pytest.mark.gpu
HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
sys.path.insert(0, os.path.join(ROOT, "examples"))


class Chain:
    """One layer over an 8-bit cache, a product with random weights, and a token of every sequence."""

    def __init__(self, seed, heads, P, lens, n_sel, V=700):
        import paper_2601_08670_gb300 as pced
        self.heads, self.lens, self.n_sel, self.V = heads, list(lens), n_sel, V
        Hq, Hkv, D = heads
        rng = np.random.default_rng(seed)
        self.rng, S = rng, len(lens)
        self.c = ref8.make_cache(rng, lens, Hkv, D, P, spare=8, spoil=False)
        # summaries of what the cache holds, so that the selection has something to go by
        self.summary = np.zeros((len(self.c["k"]), Hkv, 2, D), np.int8)
        v = ref8.values(self.c)
        self.summary = ref.summaries(dict(v, k=v["k"].float()), self.summary)
        self.cache = ref8.to_device(self.c, self.summary)
        self.rope = pced.rope_table(1e4, D, max(lens) + 16)
        dev = lambda *shape, dtype=torch.float32: torch.zeros(shape, dtype=dtype, device="cuda")
        self.qkv = dev(S, Hq + 2 * Hkv, D, dtype=torch.bfloat16)
        self.u, self.temperature = dev(S), torch.full((S,), 0.8, device="cuda")
        self.top_k = torch.tensor([0, 40] * S, dtype=torch.int32, device="cuda")[:S].contiguous()
        self.top_p, self.min_p = torch.full((S,), 0.9, device="cuda"), torch.full((S,), 0.01, device="cuda")
        mask = rng.integers(-2 ** 31, 2 ** 31, size=(S, (V + 31) // 32)).astype(np.int32)
        mask[S - 1] = 0  # a row without a token
        self.mask = torch.from_numpy(mask).cuda()
        self.weights = torch.from_numpy(rng.normal(0, 0.05, size=(Hq * D, V)).astype(np.float32)).cuda()
        self.status = dev(1, dtype=torch.int32)
        self.ws = pced.workspace(pced.paged_attention_workspace_size(S, Hq, Hkv, D), "cuda")
        self.grow = (self.cache.seq_len > 0).to(torch.int32)
        self.out = dict(q=dev(S, Hq, D, dtype=torch.bfloat16), sel=dev(S, Hkv, n_sel, dtype=torch.int32),
                        o=dev(S, Hq, D), y=dev(S, V), token=dev(S, dtype=torch.int32), logprob=dev(S))
        self.kept = ("k", "v", "scale", "summary", "seq_len")
        self.start = {n: getattr(self.cache, n).clone() for n in self.kept}

    def reset(self):
        for n, t in self.start.items():
            getattr(self.cache, n).view(torch.uint8).copy_(t.view(torch.uint8))

    def load(self, x, u):
        self.qkv.copy_(x)
        self.u.copy_(u)

    def step(self):
        import paper_2601_08670_gb300 as pced
        Hq, Hkv, _ = self.heads
        o, x = self.out, self.qkv
        self.cache.seq_len.add_(self.grow)
        pced.kv_append(self.cache, x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], rope=self.rope, q_out=o["q"],
                       status=self.status)
        pced.block_select(self.cache, o["q"], self.n_sel, sel=o["sel"], status=self.status)
        pced.paged_attention(self.cache, o["q"], sel=o["sel"], out=o["o"], ws=self.ws)
        torch.matmul(o["o"].view(len(x), -1), self.weights, out=o["y"])
        pced.logits_process(o["y"], 1, mask=self.mask, out=o["y"], status=self.status)
        pced.sample(o["y"], self.u, temperature=self.temperature, top_k=self.top_k, top_p=self.top_p, min_p=self.min_p,
                    token=o["token"], logprob=o["logprob"], status=self.status)

    def results(self):
        return [t.clone() for t in (*self.out.values(), *(getattr(self.cache, n) for n in self.kept))]

    def inputs(self, n):
        Hq, Hkv, D = self.heads
        S = len(self.lens)
        return [(ref.rng_bf16(self.rng, (S, Hq + 2 * Hkv, D)).cuda(),
                 torch.from_numpy(((self.rng.integers(0, 1 << 24, S) + 0.5) * 2.0 ** -24).astype(np.float32)).cuda())
                for _ in range(n)]


CHAINS = [((8, 2, 64), 16, [100, 700, 0, 33, 2081], 6), ((32, 8, 128), 64, [1, 64, 65, 3000], 9),
          ((14, 2, 128), 192, [191, 577], 3)]


def equal(a, b):
    return all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(a, b))


@pytest.mark.parametrize("heads,P,lens,n_sel", CHAINS)
def test_each_step_is_its_definition(cuda_ok, heads, P, lens, n_sel):
    import paper_2601_08670_gb300 as pced
    Hq, Hkv, D = heads
    ch = Chain(5, heads, P, lens, n_sel)
    c, summary, rope = ch.c, ch.summary, ch.rope.cpu().numpy()
    for x, u in ch.inputs(3):
        ch.load(x, u)
        ch.step()
        torch.cuda.synchronize()
        assert int(ch.status.item()) == 0 and pced.device_status(ch.ws) == 0
        c = dict(c, lens=[n + (n > 0) for n in c["lens"]])
        live = [s for s, n in enumerate(c["lens"]) if n]
        h = x.float().cpu().numpy()
        pos = np.array([max(n, 1) - 1 for n in c["lens"]])
        rot = ref8.rotated32(h[:, :Hq + Hkv], rope[pos])
        q = torch.from_numpy(rot[:, :Hq].copy()).to(torch.bfloat16)
        assert torch.equal(ch.out["q"].cpu()[live], q[live])
        c, summary = ref8.append(c, rot[live, Hq:], h[live, Hq + Hkv:], [int(n > 0) for n in c["lens"]], summary)
        got = ch.cache
        assert np.array_equal(got.scale.cpu().numpy(), c["scale"]) and np.array_equal(got.summary.cpu().numpy(), summary)
        for n in ("k", "v"):
            assert np.array_equal(ref8.numbers(getattr(got, n).view(torch.uint8).cpu().numpy()), ref8.numbers(c[n]))
        sel = ch.out["sel"].cpu().numpy()
        assert np.array_equal(sel[live], ref.select(c, summary, ch.out["q"], n_sel, 1, 1)[live])
        ref8.check_attention(c, ch.out["q"], ch.out["o"], sel=sel)
        y = ch.out["y"].cpu().numpy()
        for s in range(len(lens)):
            par = [float(t[s]) for t in (u, ch.temperature, ch.top_k, ch.top_p, ch.min_p)]
            token, logprob, margin = sample_ref.row(y[s], par[0], par[1], int(par[2]), par[3], par[4])
            # (a weight is off by 2^-31 at most, a sum of them too: see the operator's own tests)
            assert margin > 2.0 ** -30 and int(ch.out["token"][s]) == token
            assert token < 0 or abs(float(ch.out["logprob"][s]) - logprob) <= 2.0 ** -19 * max(1.0, abs(logprob))
        assert int(ch.out["token"][-1]) == -1


@pytest.mark.parametrize("heads,P,lens,n_sel", CHAINS)
def test_one_graph_replayed_is_the_calls(cuda_ok, heads, P, lens, n_sel):
    ch = Chain(6, heads, P, lens, n_sel)
    inputs, got = ch.inputs(4), []
    for graphed in (False, True):
        ch.reset()
        if graphed:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                ch.step()
        got.append([])
        for x in inputs:
            ch.load(*x)
            g.replay() if graphed else ch.step()
            got[-1].append(ch.results())
    torch.cuda.synchronize()
    assert int(ch.status.item()) == 0
    assert all(equal(a, b) for a, b in zip(*got))


def test_two_streams_at_once(cuda_ok):
    # two chains with caches and workspaces of their own, captured and replayed beside one another
    chains = [Chain(7 + i, *CHAINS[i]) for i in range(2)]
    inputs = [ch.inputs(1)[0] for ch in chains]
    steps, want = 6, []
    for ch, x in zip(chains, inputs):
        ch.load(*x)
        for _ in range(steps):
            ch.step()
        want.append(ch.results())
        ch.reset()
    torch.cuda.synchronize()
    graphs, streams = [], [torch.cuda.Stream() for _ in chains]
    for ch in chains:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            ch.step()
        graphs.append(g)
    torch.cuda.synchronize()
    for _ in range(steps):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for ch, w in zip(chains, want):
        assert equal(ch.results(), w)


def test_two_graphs_share_a_workspace(cuda_ok):
    # in turn on one stream: a graph of attention over all blocks, and one over a selection
    import paper_2601_08670_gb300 as pced
    ch = Chain(9, *CHAINS[0])
    ch.load(*ch.inputs(1)[0])
    ch.step()
    outs, graphs = [torch.empty_like(ch.out["o"]) for _ in range(2)], []
    sels = [None, ch.out["sel"]]
    want = [pced.paged_attention(ch.cache, ch.out["q"], sel=sel) for sel in sels]
    for sel, out in zip(sels, outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            pced.paged_attention(ch.cache, ch.out["q"], sel=sel, out=out, ws=ch.ws)
        graphs.append(g)
    for _ in range(3):
        for out in outs:
            out.fill_(float("nan"))
        for g in graphs:
            g.replay()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))


def test_the_examples_loop_over_eight_bits(cuda_ok):
    # all blocks selected is attention over all blocks; tokens drawn at a temperature near 0 are the best ones
    import paged_decode as ex
    B, N, lens = 2, 2, [7, 150, 64, 20, 97, 33]
    model = ex.Model(L=2, Hq=8, Hkv=2, D=64, V=1000, rows=max(lens) + 3)
    r = torch.tensor([[0.9, 0.2], [0.4, 0.7]], device="cuda")
    hidden = torch.randn((sum(lens), model.Hq * model.D), device="cuda", generator=torch.Generator("cuda").manual_seed(3))
    loops = [ex.Loop(model, B, N, lens, 3, torch.full((B, N), 0.5, device="cuda"), r, blocks=blocks, eight=True,
                     sampling=sampling) for blocks, sampling in ((0, None), (64, None), (0, dict(temperature=1e-6)))]
    for loop in loops:
        loop.load_documents(hidden)
        for _ in range(3):
            loop.step()
        assert loop.device_status() == 0
    dense, every, cold = loops
    assert torch.equal(dense.hidden, every.hidden) and torch.equal(dense.history, every.history)
    assert torch.equal(dense.history, cold.history)
    assert int(dense.seq_len[1]) == 153


@pytest.mark.parametrize("more", [["--eight-bit"], ["--eight-bit", "--temperature", "0.8", "--top-p", "0.95"],
                                  ["--temperature", "0.8", "--blocks", "0"]])
def test_the_example_runs(cuda_ok, more):
    res = subprocess.run([sys.executable, os.path.join(ROOT, "examples", "paged_decode.py"), "--steps", "4", *more],
                         capture_output=True, text=True, timeout=300)
    assert res.returncode == 0, res.stderr[-2000:]
    assert res.stdout.count("tokens") == 2


def test_checked_build_runs_clean_and_matches_release(cuda_ok):
    from paper_2601_08670_gb300 import build
    build.build(checked=True)
    res = subprocess.run([sys.executable, os.path.join(HERE, "decode8_checked_run.py")],
                         env=dict(os.environ, PCED_LIB="checked"), capture_output=True, text=True, timeout=600)
    assert res.returncode == 0, res.stderr[-3000:]
    checked = json.loads(res.stdout.strip().splitlines()[-1])
    assert len(checked) == len(decode8_checked_run.CASES)
    assert checked == decode8_checked_run.run_cases()
    assert all(c["status"] == 0 for c in checked)
