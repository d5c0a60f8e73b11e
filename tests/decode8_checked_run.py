"""Runs the operators over 8-bit caches and sample with whichever libpced the environment selects (PCED_LIB=checked: the
bounds-checked build) and prints, per case, the device status and a hash of the outputs as one JSON line.  Used by
test_gpu_decode8.py in a child process."""
import hashlib
import json
import os
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
sys.path[:0] = [os.path.dirname(HERE), HERE]

# (lengths, query heads, kv heads, head dim, block rows, selected blocks, vocabulary)
CASES = [([0, 1, 17, 64, 300, 2081], 8, 2, 64, 16, 4, 1000), ([700] * 40 + [5000], 32, 8, 128, 64, 9, 40001),
         ([129, 4000, 33], 28, 4, 128, 192, 7, 151936)]


def run_cases():
    import numpy as np
    import torch
    import cache8_ref as ref8
    import paged_ref as ref
    import paper_2601_08670_gb300 as pced
    out = []
    for lens, Hq, Hkv, D, P, n_sel, V in CASES:
        rng = np.random.default_rng(len(lens))
        c = ref8.make_cache(rng, lens, Hkv, D, P, spare=3)
        cache = ref8.to_device(c, np.zeros((len(c["k"]), Hkv, 2, D), np.int8))
        S = len(lens)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        ws = pced.workspace(pced.paged_attention_workspace_size(S, Hq, Hkv, D), "cuda")
        new = [min(n, P + 3) for n in lens]
        start = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device="cuda")
        qkv = ref.rng_bf16(rng, (sum(new), Hq + 2 * Hkv, D)).cuda()
        rope = pced.rope_table(1e4, D, max(lens))
        q0 = pced.kv_append(cache, qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:], rope=rope, tok_start=start,
                            status=status)
        one = ref.rng_bf16(rng, (S, Hq + 2 * Hkv, D)).cuda()
        q = pced.kv_append(cache, one[:, :Hq], one[:, Hq:Hq + Hkv], one[:, Hq + Hkv:], rope=rope, status=status)
        sel = pced.block_select(cache, q, n_sel, status=status)
        o = [pced.paged_attention(cache, q, sel=x, ws=ws) for x in (None, sel)]
        tokens = []
        for dtype in (torch.float32, torch.bfloat16):
            x = torch.from_numpy(rng.normal(0, 2.5, size=(8, V)).astype(np.float32)).to(dtype).cuda()
            x[6:] = x[6:].round()
            dev = lambda *a: torch.tensor(a, device="cuda")
            lp = torch.empty(8, device="cuda")
            tokens += [pced.sample(x, torch.linspace(0, 0.999, 8, device="cuda"), temperature=dev(0., 1., 1., 1., .7, 1., 1., 1.),
                                   top_k=dev(0, 0, 50, 700, 50, 0, 0, 600).int(), top_p=dev(1., 1., 1., 1., .9, .95, .97, 1.),
                                   min_p=dev(0., 0., 0., 0., 0., 0., 0., .01), logprob=lp, status=status), lp]
        torch.cuda.synchronize()
        h = hashlib.sha256()
        for t in (q0, q, sel, *o, *tokens, cache.k, cache.v, cache.scale, cache.summary):
            h.update(t.contiguous().view(torch.uint8).cpu().numpy().tobytes())
        out.append({"case": f"{S} {Hq}/{Hkv}/{D} {P}", "status": int(status.item()) | pced.device_status(ws),
                    "hash": h.hexdigest()[:16]})
    return out


if __name__ == "__main__":
    print(json.dumps(run_cases()))
