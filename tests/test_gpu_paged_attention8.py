"""paged_attention over 8-bit caches against softmax attention in 64 bits over the numbers that the bytes stand for: head
layouts, block sizes, lengths, selected blocks, scales of any size, and what must not matter."""
import math

import numpy as np
import pytest
import torch

import cache8_ref as ref8
import paged_ref as ref

pytestmark = pytest.mark.gpu

HEADS = [(8, 2, 64), (16, 2, 64), (28, 4, 128), (32, 8, 128), (5, 5, 64), (9, 3, 128), (6, 1, 128)]
EDGES = [0, 1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 257]


def run(c, q, sel=None, scale=None, bf16=False, total_rows=0, status=0):
    import paper_2601_08670_gb300 as pced
    S, Hq, D = q.shape
    out = torch.full((S, Hq, D), float("nan"), dtype=torch.bfloat16 if bf16 else torch.float32, device="cuda")
    lse = torch.full((S, Hq), float("nan"), device="cuda")
    ws = pced.workspace(pced.paged_attention_workspace_size(S, Hq, c["Hkv"], D), "cuda")
    cache = ref8.to_device(c)
    dsel = None if sel is None else torch.from_numpy(sel).cuda()
    for _ in range(2):  # the second call finds the workspace as the first one left it
        first = out.clone()
        pced.paged_attention(cache, q.cuda(), sel=dsel, scale=scale, out=out, lse=lse, ws=ws, total_rows=total_rows)
    torch.cuda.synchronize()
    assert torch.equal(first, out)
    assert pced.device_status(ws) == status
    return out, lse


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("P", [16, 48, 64, 192])
def test_edges_of_blocks_and_tiles(cuda_ok, heads, P):
    Hq, Hkv, D = heads
    rng = np.random.default_rng([Hq, Hkv, D, P])
    c = ref8.make_cache(rng, EDGES, Hkv, D, P)
    q = ref.rng_bf16(rng, (len(EDGES), Hq, D))
    out, lse = run(c, q)
    ref8.check_attention(c, q, out, lse)


@pytest.mark.parametrize("heads,P,lens", [
    ((32, 8, 128), 64, [5000]), ((8, 2, 64), 16, [20011]), ((28, 4, 128), 256, [4129, 32, 700]),
    ((16, 2, 64), 32, [1] * 40 + [3001, 0, 64]), ((8, 1, 128), 128, [9999, 0, 1]),
    ((32, 8, 128), 64, [0, 0, 0]), ((8, 2, 64), 64, [33] * 300), ((4, 1, 64), 256, [60_000, 3])])
def test_long_and_ragged(cuda_ok, heads, P, lens):
    Hq, Hkv, D = heads
    rng = np.random.default_rng([Hq, P, len(lens), lens[0]])
    c = ref8.make_cache(rng, lens, Hkv, D, P)
    q = ref.rng_bf16(rng, (len(lens), Hq, D))
    out, lse = run(c, q, total_rows=sum(lens))
    ref8.check_attention(c, q, out, lse)


@pytest.mark.parametrize("heads", [(8, 2, 64), (28, 4, 128), (32, 8, 128), (6, 1, 128)])
@pytest.mark.parametrize("P", [16, 48, 64, 128])
def test_selected_blocks(cuda_ok, heads, P):
    # any order, any number, a head without any, more places than blocks
    Hq, Hkv, D = heads
    rng = np.random.default_rng([Hq, P, 5])
    lens = [0, 1, P, P + 1, 5 * P - 1, 9 * P + 7, 1500]
    c = ref8.make_cache(rng, lens, Hkv, D, P)
    q = ref.rng_bf16(rng, (len(lens), Hq, D))
    n_sel = 12
    sel = np.full((len(lens), Hkv, n_sel), -1, np.int32)
    for s, n in enumerate(lens):
        nb = (n + P - 1) // P
        for h in range(Hkv):
            k = int(rng.integers(0, min(nb, n_sel) + 1))
            sel[s, h, :k] = rng.permutation(nb)[:k]
    sel[5, 0] = -1
    out, lse = run(c, q, sel=sel)
    ref8.check_attention(c, q, out, lse, sel=sel)


@pytest.mark.parametrize("heads", [(8, 2, 64), (32, 8, 128), (7, 1, 128)])
def test_scales_that_are_no_powers_of_two(cuda_ok, heads):
    Hq, Hkv, D = heads
    rng = np.random.default_rng([Hq, 6])
    c = ref8.make_cache(rng, [300, 65, 1], Hkv, D, 32, powers=False)
    q = ref.rng_bf16(rng, (3, Hq, D))
    out, lse = run(c, q)
    ref8.check_attention(c, q, out, lse)


@pytest.mark.parametrize("size", [2.0 ** -120, 2.0 ** -60, 2.0 ** -14, 1.0, 2.0 ** 15, 2.0 ** 100])
@pytest.mark.parametrize("G", [4, 7])
def test_queries_of_any_size(cuda_ok, size, G):
    # fp16 holds none of the outer ones; the cache's scales undo their size.  (Below 2^-100 a query is as 0 ... 2^-20: the
    # scores are as good as 0.)
    rng = np.random.default_rng([G, 7])
    c = ref8.make_cache(rng, [500, 70], 1, 64, 32)
    c["scale"][..., 0] = np.clip(c["scale"][..., 0].astype(np.float64) / size, 2.0 ** -100, 2.0 ** 100)
    q = torch.from_numpy((ref.rng_bf16(rng, (2, G, 64)).double().numpy() * size).astype(np.float32)).to(torch.bfloat16)
    out, lse = run(c, q)
    ref8.check_attention(c, q, out, lse)


def test_queries_with_parts_of_very_different_size(cuda_ok):
    # channels 2^-20 of the largest count where the cache's numbers make up for it; e4m3 spans 2^17.8 itself
    rng = np.random.default_rng(8)
    c = ref8.make_cache(rng, [200], 1, 128, 64)
    k = ref8.numbers(c["k"])
    k[..., ::2] *= 2.0 ** -8
    k[..., 1::2] = rng.normal(0, 100, size=k[..., 1::2].shape)
    c["k"] = ref8.to_bytes(ref8.e4m3(k))
    q = ref.rng_bf16(rng, (1, 8, 128))
    q[..., 1::2] *= 2.0 ** -20
    out, lse = run(c, q)
    ref8.check_attention(c, q, out, lse)


def test_bf16_output_and_strided_queries(cuda_ok):
    rng = np.random.default_rng(9)
    c = ref8.make_cache(rng, [70, 300, 5], 2, 64, 64)
    packed = ref.rng_bf16(rng, (3, 12, 64)).cuda()  # queries beside something else
    q = packed[:, :8]
    assert not q.is_contiguous()
    out, lse = run(c, q, bf16=True)
    ref8.check_attention(c, q, out, lse, bf16=True)


@pytest.mark.parametrize("scale", [0.0, 3.0, -0.2])
def test_softmax_scales(cuda_ok, scale):
    # flat, peaked (one key takes nearly all) and negative
    rng = np.random.default_rng(10)
    c = ref8.make_cache(rng, [400, 64, 3], 2, 128, 64)
    q = ref.rng_bf16(rng, (3, 8, 128))
    out, lse = run(c, q, scale=scale)
    ref8.check_attention(c, q, out, lse, scale=scale)


@pytest.mark.parametrize("P", [16, 64])
@pytest.mark.parametrize("G", [2, 8])
def test_every_byte_is_read_as_its_number(cuda_ok, G, P):
    # one row a sequence: the output is the value; one channel of the key holds each number, the score shows in lse
    import paper_2601_08670_gb300 as pced
    b = np.arange(256, dtype=np.uint8)
    n = ref8.numbers(b)
    kk, v = np.zeros((256, 1, P, 64), np.uint8), np.zeros((256, 1, P, 64), np.uint8)
    kk[:, 0, 0, 5], v[:, 0, 0] = b, b[:, None]
    t = lambda a: torch.from_numpy(a).cuda()
    cache = pced.PagedCache8(t(kk).view(torch.float8_e4m3fn), t(v).view(torch.float8_e4m3fn),
                             torch.tensor([0.5, 2.0], device="cuda").repeat(256, 1, 1),
                             torch.arange(256, dtype=torch.int32, device="cuda")[:, None].contiguous(),
                             torch.ones(256, dtype=torch.int32, device="cuda"))
    q = torch.zeros((256, G, 64), dtype=torch.bfloat16, device="cuda")
    q[:, :, 5] = 1.0
    lse = torch.empty((256, G), device="cuda")
    out = pced.paged_attention(cache, q, scale=1.0, lse=lse).cpu().numpy()
    fine = ~np.isnan(n)
    # (the probability is exp2 of a difference that is 0 but for the fp32 product of log2(e) and the score)
    assert np.allclose(out[fine], 2 * n[fine, None, None], rtol=2.0 ** -20, atol=0)
    assert np.isnan(out[~fine]).all()
    assert np.allclose(lse.cpu().numpy()[fine], 0.5 * n[fine, None], rtol=2.0 ** -20, atol=2.0 ** -20)


def test_bad_table_entries_and_numbers_are_left_out(cuda_ok):
    import paper_2601_08670_gb300 as pced
    rng = np.random.default_rng(11)
    P, lens = 64, [300, 200]
    c = ref8.make_cache(rng, lens, 2, 64, P)
    q = ref.rng_bf16(rng, (2, 8, 64))
    c["table"][0, 2] = len(c["k"])  # one past the pool
    out, lse = run(c, q, status=pced.PCED_DEV_BAD_BLOCK)
    sel = np.tile(np.array([0, 1, 3, 4, -1], np.int32), (2, 2, 1))
    sel[1] = [0, 1, 2, 3, -1]  # all of the other sequence's
    c["table"][0, 2] = 0  # (not read by the reference either)
    ref8.check_attention(c, q, out, lse, sel=sel)
    bad = sel.copy()
    bad[0, 0, 4], bad[1, 1, 4] = 5, -2  # block 5 holds no live row
    out, lse = run(c, q, sel=bad, status=pced.PCED_DEV_BAD_BLOCK)
    ref8.check_attention(c, q, out, lse, sel=sel)


def test_bad_lengths_are_clipped_and_flagged(cuda_ok):
    import paper_2601_08670_gb300 as pced
    rng = np.random.default_rng(12)
    c = ref8.make_cache(rng, [64, 128], 2, 64, 64, spoil=False)
    c["table"] = c["table"][:, :2].copy()
    q = ref.rng_bf16(rng, (2, 8, 64))
    c["lens"] = np.array([-5, 129], np.int32)
    out, lse = run(c, q, status=pced.PCED_DEV_BAD_LENGTH)
    c["lens"] = np.array([0, 128], np.int32)
    ref8.check_attention(c, q, out, lse)


def test_rows_beyond_32_bit_offsets(cuda_ok):
    # pools of more than 2^32 bytes; the used blocks lie at their ends
    import paper_2601_08670_gb300 as pced
    rng = np.random.default_rng(13)
    Hkv, P, D, n = 8, 64, 128, 700
    nb = 2 ** 32 // (Hkv * P * D) + 40
    small = ref8.make_cache(rng, [n], Hkv, D, P)
    pools = []
    for x in ("k", "v"):
        big = torch.empty((nb, Hkv, P, D), dtype=torch.uint8, device="cuda")
        big[-len(small[x]):] = torch.from_numpy(small[x]).cuda()
        pools.append(big.view(torch.float8_e4m3fn))
    scale = torch.full((nb, Hkv, 2), float("nan"), device="cuda")
    scale[-len(small["k"]):] = torch.from_numpy(small["scale"]).cuda()
    table = torch.from_numpy(small["table"] + np.int32(nb - len(small["k"]))).cuda()
    cache = pced.PagedCache8(*pools, scale, table, torch.tensor([n], dtype=torch.int32, device="cuda"))
    q = ref.rng_bf16(rng, (1, 32, D))
    out = pced.paged_attention(cache, q.cuda())
    ref8.check_attention(small, q, out)


def test_another_stream_and_graph_replays(cuda_ok):
    import paper_2601_08670_gb300 as pced
    rng = np.random.default_rng(14)
    c = ref8.make_cache(rng, [2000, 31, 0], 8, 128, 64)
    q = ref.rng_bf16(rng, (3, 32, 128))
    cache, dq = ref8.to_device(c), q.cuda()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = pced.paged_attention(cache, dq, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    ref8.check_attention(c, q, out)
    ws = pced.workspace(pced.paged_attention_workspace_size(3, 32, 8, 128), "cuda")
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        pced.paged_attention(cache, dq, ws=ws, out=out)
    for _ in range(3):
        out.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        ref8.check_attention(c, q, out)


# What is left of a probability that is held to 23 bits.  Of o = p v / (1 + p), relative: the score is a whole number times
# one rounded constant (two roundings of |x| <= 2.9, 2.4e-7 after the exponential), exp2 (two units, 2.4e-7), two parts of
# which the second is off by 2^-12 of 2^-12 (6e-8), products of the parts joined (2^-23, 1.2e-7), the sum, its reciprocal
# and the last product (2^-24 each, 1.8e-7): below 1e-6.
@pytest.mark.parametrize("heads", [(4, 1, 64), (8, 2, 128), (8, 1, 64), (7, 1, 128)])
def test_probabilities_keep_23_bits(cuda_ok, heads):
    import paper_2601_08670_gb300 as pced
    Hq, Hkv, D = heads
    S, P = 128, 16
    # two rows: one that scores 0, whose value is 0, and one that scores -i (16 a and the rest b, in two channels)
    i = np.arange(S)
    k = np.zeros((S, Hkv, P, D))
    k[:, :, 1, 3], k[:, :, 1, 4] = -(i // 16)[:, None], -(i % 16)[:, None]
    v = np.zeros((S, Hkv, P, D))
    v[:, :, 1] = 1.0
    q = torch.zeros((S, Hq, D), dtype=torch.bfloat16, device="cuda")
    q[:, :, 3], q[:, :, 4] = 16.0, 1.0
    t = lambda a: torch.from_numpy(ref8.to_bytes(a)).cuda().view(torch.float8_e4m3fn)
    cache = pced.PagedCache8(t(k), t(v), torch.ones((S, Hkv, 2), device="cuda"),
                             torch.arange(S, dtype=torch.int32, device="cuda")[:, None].contiguous(),
                             torch.full((S,), 2, dtype=torch.int32, device="cuda"))
    out = pced.paged_attention(cache, q, scale=1 / 64).double().cpu().numpy()
    p = np.exp(-i / 64)[:, None, None]
    assert np.abs(out / (p / (1 + p)) - 1).max() <= 1e-6


def test_weights_far_below_the_reference_count(cuda_ok):
    # 2^17 rows that each have 2^-28 of the first one's weight (216 is between two e4m3 numbers and becomes 224): in fp16
    # alone they would be nothing.  Their sum is 2^-11 of the output; relative to it the bound is that of the sums: 2^-20
    import paper_2601_08670_gb300 as pced
    P, n = 256, 1 + 2 ** 17
    nb = (n + P - 1) // P
    k, v = np.zeros((nb, 1, P, 64)), np.zeros((nb, 1, P, 64))
    k[..., 0] = -27.0 * 8
    k[0, 0, 0, 0] = 0.0
    v[...] = 1.0
    v[0, 0, 0] = 0.0
    k = ref8.e4m3(k)
    t = lambda a: torch.from_numpy(ref8.to_bytes(a)).cuda().view(torch.float8_e4m3fn)
    cache = pced.PagedCache8(t(k), t(v), torch.ones((nb, 1, 2), device="cuda"),
                             torch.arange(nb, dtype=torch.int32, device="cuda")[None].contiguous(),
                             torch.tensor([n], dtype=torch.int32, device="cuda"))
    for G in (4, 8):
        q = torch.zeros((1, G, 64), dtype=torch.bfloat16, device="cuda")
        q[..., 0] = 1.0
        out = pced.paged_attention(cache, q, scale=math.log(2) / 8).double().cpu().numpy()
        w = (n - 1) * 2.0 ** (k[1, 0, 0, 0] / 8)
        # (the scale is rounded to fp32: 28 of 2^-24, times ln 2, in the exponent)
        assert np.abs(out / (w / (1 + w)) - 1).max() <= 28 * 2.0 ** -24 + 2.0 ** -20
