"""Runs the operators over paged caches with whichever libpced the environment selects (PCED_LIB=checked: the
bounds-checked build) and prints, per case, the device status and a hash of the outputs as one JSON line.  Used by
test_gpu_paged_checked.py in a child process."""
import hashlib
import json
import os
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
sys.path[:0] = [os.path.dirname(HERE), HERE]

# (lengths, query heads, kv heads, head dim, block rows, selected blocks)
CASES = [([0, 1, 17, 64, 300, 2081], 8, 2, 64, 16, 4), ([700] * 40 + [5000], 32, 8, 128, 64, 9),
         ([129, 4000, 33], 28, 4, 128, 192, 7)]


def run_cases():
    import numpy as np
    import torch
    import paged_ref as ref
    import paper_2601_08670_gb300 as pced
    out = []
    for lens, Hq, Hkv, D, P, n_sel in CASES:
        rng = np.random.default_rng(len(lens))
        c = ref.make_cache(rng, lens, Hkv, D, P, spare=3)
        cache = ref.to_device(c, np.zeros((len(c["k"]), Hkv, 2, D), np.int8))
        S = len(lens)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        ws = pced.workspace(pced.paged_attention_workspace_size(S, Hq, Hkv, D), "cuda")
        pced.block_summaries(cache, status=status)
        new = [min(n, 3) for n in lens]
        start = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device="cuda")
        qkv = ref.rng_bf16(rng, (sum(new), Hq + 2 * Hkv, D)).cuda()
        rope = pced.rope_table(1e4, D, max(lens))
        q0 = pced.kv_append(cache, qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:], rope=rope, tok_start=start,
                            status=status)
        one = ref.rng_bf16(rng, (S, Hq + 2 * Hkv, D)).cuda()
        q = pced.kv_append(cache, one[:, :Hq], one[:, Hq:Hq + Hkv], one[:, Hq + Hkv:], rope=rope, status=status)
        sel = pced.block_select(cache, q, n_sel, status=status)
        o = [pced.paged_attention(cache, q, sel=x, ws=ws) for x in (None, sel)]
        x = torch.from_numpy(rng.normal(size=(2 * S, 3001)).astype(np.float32)).cuda()
        y = pced.logits_process(x, 2, history=sel[:, 0].clamp(min=0).contiguous(),
                                history_len=torch.full((S,), n_sel, dtype=torch.int32, device="cuda"),
                                penalties=torch.full((S, 3), 1.1, device="cuda"), status=status)
        torch.cuda.synchronize()
        h = hashlib.sha256()
        for t in (q0, q, sel, *o, y, cache.k, cache.v, cache.summary):
            h.update(t.cpu().contiguous().view(torch.uint8).numpy().tobytes())
        out.append({"case": f"{S} {Hq}/{Hkv}/{D} {P}", "status": int(status.item()) | pced.device_status(ws),
                    "hash": h.hexdigest()[:16]})
    return out


if __name__ == "__main__":
    print(json.dumps(run_cases()))
