"""paged_attention against softmax attention in 64 bits: head layouts, block sizes, lengths from none to long ones,
selected blocks, idle sequences, strides, and what must not matter (rows past the live ones, other streams)."""
import numpy as np
import pytest
import torch

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
    cache = ref.to_device(c)
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
    c = ref.make_cache(rng, EDGES, Hkv, D, P)
    q = ref.rng_bf16(rng, (len(EDGES), Hq, D))
    out, lse = run(c, q)
    ref.check_attention(c, q, out, lse)


@pytest.mark.parametrize("heads,P,lens", [
    ((32, 8, 128), 64, [5000]), ((8, 2, 64), 16, [20011]), ((28, 4, 128), 256, [4129, 32, 700]),
    ((16, 2, 64), 32, [1] * 40 + [3001, 0, 64]), ((8, 1, 128), 128, [9999, 0, 1]),
    ((32, 8, 128), 64, [0, 0, 0]), ((8, 2, 64), 64, [33] * 300)])
def test_long_and_ragged(cuda_ok, heads, P, lens):
    Hq, Hkv, D = heads
    rng = np.random.default_rng([Hq, P, len(lens), lens[0]])
    c = ref.make_cache(rng, lens, Hkv, D, P)
    q = ref.rng_bf16(rng, (len(lens), Hq, D))
    out, lse = run(c, q, total_rows=sum(lens))
    ref.check_attention(c, q, out, lse)


@pytest.mark.parametrize("heads", [(8, 2, 64), (28, 4, 128), (32, 8, 128), (6, 1, 128)])
@pytest.mark.parametrize("P", [16, 48, 64, 128])
def test_selected_blocks(cuda_ok, heads, P):
    # any order, any number, a head without any, more places than blocks
    Hq, Hkv, D = heads
    rng = np.random.default_rng([Hq, P, 5])
    lens = [0, 1, P, P + 1, 5 * P - 1, 9 * P + 7, 1500]
    c = ref.make_cache(rng, lens, Hkv, D, P)
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
    ref.check_attention(c, q, out, lse, sel=sel)


def test_many_selected_blocks_split_over_ctas(cuda_ok):
    rng = np.random.default_rng(8)
    lens, P = [30_000, 11_111], 32
    c = ref.make_cache(rng, lens, 4, 128, P)
    q = ref.rng_bf16(rng, (2, 28, 128))
    sel = np.stack([np.stack([np.sort(rng.permutation((n + P - 1) // P)[:300]) for _ in range(4)]) for n in lens])
    out, lse = run(c, q, sel=sel.astype(np.int32))
    ref.check_attention(c, q, out, lse, sel=sel)


def test_bf16_output_and_strided_queries(cuda_ok):
    rng = np.random.default_rng(9)
    c = ref.make_cache(rng, [70, 300, 5], 2, 64, 64)
    packed = ref.rng_bf16(rng, (3, 12, 64)).cuda()  # queries beside something else
    q = packed[:, :8]
    assert not q.is_contiguous()
    out, lse = run(c, q, bf16=True)
    ref.check_attention(c, q, out, lse, bf16=True)


@pytest.mark.parametrize("scale", [0.0, 3.0, -0.2])
def test_scales(cuda_ok, scale):
    # flat, peaked (one key takes nearly all) and negative
    rng = np.random.default_rng(10)
    c = ref.make_cache(rng, [400, 64, 3], 2, 128, 64)
    q = ref.rng_bf16(rng, (3, 8, 128))
    out, lse = run(c, q, scale=scale)
    ref.check_attention(c, q, out, lse, scale=scale)


def test_bad_table_entries_and_numbers_are_left_out(cuda_ok):
    import paper_2601_08670_gb300 as pced
    rng = np.random.default_rng(11)
    P, lens = 64, [300, 200]
    c = ref.make_cache(rng, lens, 2, 64, P)
    q = ref.rng_bf16(rng, (2, 8, 64))
    c["table"][0, 2] = len(c["k"])  # one past the pool
    out, lse = run(c, q, status=pced.PCED_DEV_BAD_BLOCK)
    sel = np.tile(np.array([0, 1, 3, 4, -1], np.int32), (2, 2, 1))
    sel[1] = [0, 1, 2, 3, -1]  # all of the other sequence's
    c["table"][0, 2] = 0  # (not read by the reference either)
    ref.check_attention(c, q, out, lse, sel=sel)
    bad = sel.copy()
    bad[0, 0, 4], bad[1, 1, 4] = 5, -2  # block 5 holds no live row
    out, lse = run(c, q, sel=bad, status=pced.PCED_DEV_BAD_BLOCK)
    ref.check_attention(c, q, out, lse, sel=sel)


def test_bad_lengths_are_clipped_and_flagged(cuda_ok):
    import paper_2601_08670_gb300 as pced
    rng = np.random.default_rng(12)
    c = ref.make_cache(rng, [64, 128], 2, 64, 64, spoil=False)
    c["table"] = c["table"][:, :2].copy()
    q = ref.rng_bf16(rng, (2, 8, 64))
    c["lens"] = np.array([-5, 129], np.int32)
    out, lse = run(c, q, status=pced.PCED_DEV_BAD_LENGTH)
    c["lens"] = np.array([0, 128], np.int32)
    ref.check_attention(c, q, out, lse)


def test_rows_beyond_32_bit_offsets(cuda_ok):
    # a pool of more than 2^32 bytes and 2^31 elements; the used blocks lie at its end
    import paper_2601_08670_gb300 as pced
    rng = np.random.default_rng(13)
    Hkv, P, D, n = 8, 64, 128, 700
    nb = 2 ** 31 // (Hkv * P * D) + 40
    small = ref.make_cache(rng, [n], Hkv, D, P)
    used = small["table"][0, :(n + P - 1) // P]
    pools = []
    for x in ("k", "v"):
        big = torch.empty((nb, Hkv, P, D), dtype=torch.bfloat16, device="cuda")
        big[-len(small[x]):] = small[x].cuda()
        pools.append(big)
    table = torch.from_numpy(small["table"] + np.int32(nb - len(small["k"]))).cuda()
    cache = pced.PagedCache(*pools, table, torch.tensor([n], dtype=torch.int32, device="cuda"))
    q = ref.rng_bf16(rng, (1, 32, D))
    out = pced.paged_attention(cache, q.cuda())
    ref.check_attention(small, q, out)
    assert int(used.max()) < len(small["k"])


def test_another_stream(cuda_ok):
    # inputs made on the current stream, the call on another one, which waits for it
    import paper_2601_08670_gb300 as pced
    rng = np.random.default_rng(14)
    c = ref.make_cache(rng, [2000, 31], 8, 128, 64)
    q = ref.rng_bf16(rng, (2, 32, 128))
    cache, dq = ref.to_device(c), q.cuda()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = pced.paged_attention(cache, dq, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    ref.check_attention(c, q, out)


def test_graph_replays(cuda_ok):
    import paper_2601_08670_gb300 as pced
    rng = np.random.default_rng(15)
    c = ref.make_cache(rng, [900, 31, 0], 2, 64, 64)
    q = ref.rng_bf16(rng, (3, 8, 64))
    cache, dq = ref.to_device(c), q.cuda()
    ws = pced.workspace(pced.paged_attention_workspace_size(3, 8, 2, 64), "cuda")
    out = pced.paged_attention(cache, dq, ws=ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        pced.paged_attention(cache, dq, ws=ws, out=out)
    for _ in range(3):
        out.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        ref.check_attention(c, q, out)


def test_agrees_with_slab_attention(cuda_ok):
    import paper_2601_08670_gb300 as pced
    rng = np.random.default_rng(16)
    Hq, Hkv, D, P, n = 32, 8, 128, 64, 500
    c = ref.make_cache(rng, [n], Hkv, D, P)
    q = ref.rng_bf16(rng, (1, Hq, D))
    out, _ = run(c, q)
    rows = np.arange(n)
    slab = [torch.stack([c[x][c["table"][0, rows // P], h, rows % P] for h in range(Hkv)]).cuda() for x in ("k", "v")]
    one = torch.tensor([n], dtype=torch.int32, device="cuda")
    want = pced.decode_attention(q.cuda(), *slab, torch.zeros(1, dtype=torch.int64, device="cuda"), one, one, Hkv, n)
    _, _, tol, _ = ref.attention(c, q)
    assert np.all(np.abs(ref.f64(out) - ref.f64(want)).max(axis=2) <= 2 * tol)


@pytest.mark.parametrize("heads", [(8, 2, 64), (16, 2, 64), (32, 8, 128), (28, 4, 128), (5, 5, 64)])
def test_segments_of_one_tile_among_longer_ones(cuda_ok, heads):
    # a warpgroup finishes a segment of one tile by itself, both meet for longer ones: every order of the two, idle
    # sequences between them, and enough of them that a CTA holds many
    Hq, Hkv, D = heads
    rng = np.random.default_rng([Hq, 21])
    lens = [int(x) for x in rng.choice([0, 1, 5, 17, 33, 64, 65, 100, 128, 129, 200], size=500)]
    c = ref.make_cache(rng, lens, Hkv, D, 64)
    q = ref.rng_bf16(rng, (len(lens), Hq, D))
    out, lse = run(c, q)
    ref.check_attention(c, q, out, lse)


@pytest.mark.parametrize("heads,n", [((4, 1, 64), 60_000), ((1, 1, 128), 30_000), ((8, 1, 128), 30_000), ((7, 1, 64), 12_000)])
def test_one_segment_over_all_ctas(cuda_ok, heads, n):
    # so many records that their merge is shared among the threads
    Hq, Hkv, D = heads
    rng = np.random.default_rng([Hq, n])
    c = ref.make_cache(rng, [n, 3], Hkv, D, 256)
    q = ref.rng_bf16(rng, (2, Hq, D))
    out, lse = run(c, q)
    ref.check_attention(c, q, out, lse)
