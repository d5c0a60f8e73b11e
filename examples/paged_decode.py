"""A decode loop with layers of its own over paged caches.

The experts of a query (documents, and the amateur without one) decode as one
batch, each over its own paged cache, as `Decoder` does; here the layers are
the program's: rotary attention layers with random weights, PyTorch's matrix
products between the library's operators.

    documents   kv_append of whole sequences, block_summaries
    each layer  kv_append -> block_select -> paged_attention
    each token  lm_head_logprobs -> logits_process -> contrastive_select, with the rows made logits again
                before logits_process and normalised after it

Run: python examples/paged_decode.py [--steps 8] [--blocks 8]
"""
import argparse
import math
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

import paper_2601_08670_gb300 as pced

RMS_EPS = 1e-6


def rmsnorm(x):
    return (x * torch.rsqrt(x.square().mean(-1, keepdim=True) + RMS_EPS)).to(torch.bfloat16)


class Model:
    """L attention layers: x += attention(rmsnorm(x) Wqkv) Wo."""

    def __init__(self, L, Hq, Hkv, D, V, rows, theta=1e4, seed=0, device="cuda"):
        self.L, self.Hq, self.Hkv, self.D, self.V = L, Hq, Hkv, D, V
        d = Hq * D
        g = torch.Generator(device=device).manual_seed(seed)

        def weights(*shape):
            return torch.empty(shape, dtype=torch.bfloat16, device=device).normal_(0, shape[-1] ** -0.5, generator=g)

        self.embed = torch.empty((V, d), dtype=torch.bfloat16, device=device).normal_(0, 1, generator=g)
        self.qkv = [weights((Hq + 2 * Hkv) * D, d) for _ in range(L)]
        self.out = [weights(d, d) for _ in range(L)]
        self.unembed = weights(V, d)
        self.rope = pced.rope_table(theta, D, rows, device)

    def project(self, layer, x):
        """q, k, v of x [T, d]: three parts of one product's output, which the append takes as they lie."""
        y = (rmsnorm(x) @ self.qkv[layer].T).view(-1, self.Hq + 2 * self.Hkv, self.D)
        return y[:, :self.Hq], y[:, self.Hq:self.Hq + self.Hkv], y[:, self.Hq + self.Hkv:]


class Loop:
    """B queries of N experts and the amateur; `blocks` 0: attention over all blocks, else over so many."""

    def __init__(self, model, B, N, lens, max_steps, beta, r, gamma=2.5, block_rows=16, blocks=0, penalties=None,
                 mask=None):
        m, dev = model, model.embed.device
        self.model, self.B, self.N, self.blocks, self.gamma = m, B, N, blocks, gamma
        S = B * (N + 1)
        need = [(n + max_steps + block_rows - 1) // block_rows for n in lens]
        table = torch.full((S, max(need)), -1, dtype=torch.int32)
        order = torch.randperm(sum(need), generator=torch.Generator().manual_seed(1)).to(torch.int32)
        at = 0
        for s, n in enumerate(need):
            table[s, :n] = order[at:at + n]
            at += n
        self.seq_len = torch.tensor(lens, dtype=torch.int32, device=dev)
        table = table.to(dev)
        # the largest key a step of the summaries stands for; keys are sums of d products of unit variance
        step = torch.full((m.Hkv,), 5.0 / 127.0, device=dev)

        def pool(dtype, *tail):
            return torch.zeros((sum(need), m.Hkv, *tail), dtype=dtype, device=dev)

        self.caches = [pced.PagedCache(pool(torch.bfloat16, block_rows, m.D), pool(torch.bfloat16, block_rows, m.D),
                                       table, self.seq_len, summary=pool(torch.int8, 2, m.D), key_step=step)
                       for _ in range(m.L)]
        self.status = torch.zeros(1, dtype=torch.int32, device=dev)
        self.ws = pced.workspace(pced.paged_attention_workspace_size(S, m.Hq, m.Hkv, m.D), dev)
        self.beta, self.r = beta, r
        self.history = torch.full((B, max_steps), -1, dtype=torch.int32, device=dev)
        self.expert = torch.zeros((B, max_steps), dtype=torch.int32, device=dev)
        self.t = 0
        self.n_history = torch.zeros(B, dtype=torch.int32, device=dev)
        self.penalties, self.mask = penalties, mask

    def load_documents(self, hidden):
        """Fill the caches from hidden states [sum(lens), d], the sequences one after another (what an offline
        encoder would have stored); appended in one call per layer."""
        lens = self.seq_len.cpu()
        start = torch.cat([torch.zeros(1, dtype=torch.int32), lens.cumsum(0).to(torch.int32)]).to(hidden.device)
        for layer, cache in enumerate(self.caches):
            _, k, v = self.model.project(layer, hidden)
            pced.kv_append(cache, None, k, v, rope=self.model.rope, tok_start=start, status=self.status)
            pced.block_summaries(cache, status=self.status)  # (kv_append has made them; a cache loaded as it is needs this)

    def step(self):
        m, S = self.model, self.B * (self.N + 1)
        last = self.history[:, self.t - 1] if self.t else torch.zeros(self.B, dtype=torch.int32,
                                                                      device=self.seq_len.device)
        x = m.embed[last.long()].float().repeat_interleave(self.N + 1, 0)
        self.seq_len += 1
        for layer, cache in enumerate(self.caches):
            q, k, v = m.project(layer, x)
            q = pced.kv_append(cache, q, k, v, rope=m.rope, status=self.status)
            sel = pced.block_select(cache, q, self.blocks, status=self.status) if self.blocks else None
            o = torch.empty((S, m.Hq, m.D), dtype=torch.bfloat16, device=x.device)
            pced.paged_attention(cache, q, sel=sel, out=o, ws=self.ws)
            x = x + (o.view(S, -1) @ m.out[layer].T).float()
        self.hidden = rmsnorm(x)
        lp, lse = pced.lm_head_logprobs(self.hidden, m.unembed)
        if self.penalties is not None or self.mask is not None:
            use = self.penalties is not None
            z = lp.add_(lse[:, None])  # logits: a penalty asks for their sign
            pced.logits_process(z, self.N + 1, history=self.history if use else None,
                                history_len=self.n_history if use else None, penalties=self.penalties,
                                mask=self.mask, out=z, status=self.status)
            lp = z.log_softmax(1)  # (a mask that forbids everything leaves no distribution)
        self.logprobs = lp
        token, expert, _ = pced.contrastive_select(lp, self.beta, self.r, self.gamma)
        self.history[:, self.t], self.expert[:, self.t] = token, expert
        self.n_history += 1
        self.t += 1
        return token, expert

    def device_status(self):
        return int(self.status.item()) | pced.device_status(self.ws)


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=8)
    ap.add_argument("--blocks", type=int, default=8, help="blocks that attention reads (0: all)")
    args = ap.parse_args()
    torch.manual_seed(0)
    B, N = 2, 3
    lens = [32 if j == 0 else 200 + 57 * j for _ in range(B) for j in range(N + 1)]
    model = Model(L=4, Hq=8, Hkv=2, D=64, V=8192, rows=max(lens) + args.steps)
    beta = torch.full((B, N), 0.5, device="cuda")
    r = torch.rand((B, N), device="cuda")
    loop = Loop(model, B, N, lens, args.steps, beta, r, blocks=args.blocks,
                penalties=torch.tensor([[1.1, 0.2, 0.2]] * B, device="cuda"))
    loop.load_documents(torch.randn((sum(lens), model.Hq * model.D), device="cuda"))
    for _ in range(args.steps):
        loop.step()
    if loop.device_status():
        raise RuntimeError(f"device status {loop.device_status():#x}")
    for b in range(B):
        print(f"query {b}: tokens {loop.history[b].tolist()} experts {loop.expert[b].tolist()}")


if __name__ == "__main__":
    main()
