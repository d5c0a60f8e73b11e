"""kv_append and block_summaries: rows, rotation and summaries against the definition, and what stays untouched."""
import numpy as np
import pytest
import torch

import paged_ref as ref

pytestmark = pytest.mark.gpu


def table_of(rows, D, theta=1e4):
    import paper_2601_08670_gb300 as pced
    return pced.rope_table(theta, D, rows)


def expected_close(got, want, x):
    """bf16 roundings (2^-9 of the value) of fp32 products and sums (2^-24 each of the terms)."""
    assert np.all(np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -22 * np.abs(x).max() + 1e-38)


def run(lens, new, heads, P, rope=True, positions=None, one=False, spare=5, seed=0, old_summary=None, q_none=False,
        packed=True):
    """Appends and checks everything; returns the device status."""
    import paper_2601_08670_gb300 as pced
    Hq, Hkv, D = heads
    rng = np.random.default_rng([seed, Hq, P, len(lens)])
    c = ref.make_cache(rng, lens, Hkv, D, P, spare=spare, spoil=False)
    nb = len(c["k"])
    summ = rng.integers(-60, 61, size=(nb, Hkv, 2, D)).astype(np.int8)
    cache = ref.to_device(c, summ)
    T = sum(new)
    qkv = ref.rng_bf16(rng, (T, Hq + 2 * Hkv, D), 1.5)
    dev = qkv.cuda()
    q, k, v = dev[:, :Hq], dev[:, Hq:Hq + Hkv], dev[:, Hq + Hkv:]
    if not packed:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    seq = np.repeat(np.arange(len(lens)), new)
    row = np.concatenate([np.arange(n - m, n) for n, m in zip(lens, new)]).astype(np.int64)
    pos = row if positions is None else positions
    rows = int(pos.max()) + 1
    tab = table_of(rows, D) if rope else None
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    q_out = pced.kv_append(cache, None if q_none else q, k, v, rope=tab,
                           tok_start=None if one else torch.from_numpy(start).cuda(),
                           positions=None if positions is None else torch.from_numpy(pos.astype(np.int32)).cuda(),
                           status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    x = ref.f64(qkv)
    rot = x[:, :Hq + Hkv]
    if rope:
        rot = ref.rotate(rot, tab.cpu().numpy().astype(np.float64)[pos])
    if q_none:
        assert q_out is None
    else:
        expected_close(ref.f64(q_out), rot[:, :Hq], x)
    want_k, want_v = c["k"].clone(), c["v"].clone()
    b, at = c["table"][seq, row // P], row % P
    got_k, got_v = cache.k.cpu(), cache.v.cpu()
    expected_close(ref.f64(got_k[b, :, at]), rot[:, Hq:], x)
    want_k[b, :, at] = got_k[b, :, at]  # (checked above)
    want_v[b, :, at] = qkv[:, Hq + Hkv:]
    assert torch.equal(got_k.view(torch.int16), want_k.view(torch.int16))
    assert torch.equal(got_v.view(torch.int16), want_v.view(torch.int16))
    # summaries follow the stored keys
    want = summ.copy()
    stored = got_k.float().numpy()
    for s in range(len(lens)):
        for j in sorted({int(r) // P for r in row[seq == s]}):
            r = np.array([i for i in row[seq == s] if i // P == j]) % P
            blk = c["table"][s, j]
            for h in range(Hkv):
                nw = ref.bounds(stored[blk, h, r], c["key_step"][h])
                want[blk, h] = nw if 0 in r else np.stack([np.maximum(nw[0], summ[blk, h, 0]),
                                                           np.minimum(nw[1], summ[blk, h, 1])])
    assert np.array_equal(cache.summary.cpu().numpy(), want)


HEADS = [(8, 2, 64), (16, 2, 64), (28, 4, 128), (32, 8, 128), (3, 3, 64)]


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("P", [16, 64, 192])
def test_one_token_per_sequence(cuda_ok, heads, P):
    lens = [1, 2, 16, 17, 64, 65, 192, 193, 700]
    run(lens, [1] * len(lens), heads, P, one=True)
    run(lens, [1] * len(lens), heads, P, one=False, rope=False)


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("P", [16, 64, 256])
def test_ragged_prompts(cuda_ok, heads, P):
    # whole sequences, parts that begin and end inside blocks, sequences without tokens
    lens = [0, 1, 63, 64, 65, 300, 129, 40, 500]
    new = [0, 1, 63, 64, 65, 300, 100, 0, 7]
    run(lens, new, heads, P, packed=P != 64)


def test_many_sequences_and_one_long_prompt(cuda_ok):
    run([5] * 700, [2] * 700, (8, 2, 64), 16)
    run([3000], [2900], (8, 2, 64), 256, packed=False)


def test_positions_of_their_own(cuda_ok):
    run([10, 20, 30], [3, 20, 1], (8, 2, 64), 16, positions=np.arange(24) * 37 % 101)


def test_keys_without_queries(cuda_ok):
    run([10, 20, 30], [3, 20, 1], (2, 2, 64), 16, q_none=True)


def test_idle_sequences_get_no_token(cuda_ok):
    import paper_2601_08670_gb300 as pced
    rng = np.random.default_rng(1)
    lens = [5, 0, 70]
    c = ref.make_cache(rng, lens, 2, 64, 64, spoil=False)
    cache = ref.to_device(c, np.zeros((len(c["k"]), 2, 2, 64), np.int8))
    x = ref.rng_bf16(rng, (3, 12, 64)).cuda()
    q_out = torch.full((3, 8, 64), float("nan"), dtype=torch.bfloat16, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    pced.kv_append(cache, x[:, :8], x[:, 8:10], x[:, 10:], q_out=q_out, status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    assert torch.equal(q_out[[0, 2]], x[[0, 2], :8]) and not q_out[1].any()
    b = c["table"][1, 0]
    assert torch.equal(cache.k[b].cpu(), c["k"][b]) and not cache.summary[int(b)].any()


def append_flags(change, T=3, one=False, rope_rows=0):
    """Device status of an append whose cache, starts or positions `change` edits; nothing else may change."""
    import paper_2601_08670_gb300 as pced
    rng = np.random.default_rng(2)
    lens = [5, 20, 70]
    d = dict(c=ref.make_cache(rng, lens, 2, 64, 64, spoil=False), start=np.arange(4, dtype=np.int32),
             pos=np.zeros(3, np.int32))
    change(d)
    c = d["c"]
    cache = ref.to_device(c, np.zeros((len(c["k"]), 2, 2, 64), np.int8))
    x = ref.rng_bf16(rng, (T, 12, 64)).cuda()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    rope = table_of(rope_rows, 64) if rope_rows else None
    q = pced.kv_append(cache, x[:, :8], x[:, 8:10], x[:, 10:], rope=rope,
                       tok_start=None if one else torch.from_numpy(d["start"]).cuda(),
                       positions=torch.from_numpy(d["pos"]).cuda() if rope_rows else None, status=status)
    torch.cuda.synchronize()
    return int(status.item()), c, cache, x, q


def changed_blocks(c, cache):
    return set(np.unique(np.nonzero((cache.v.cpu() != c["v"]).flatten(1).any(1).numpy())[0]).tolist())


def test_bad_counts_leave_the_sequence_out(cuda_ok):
    import paper_2601_08670_gb300 as pced
    for change in (lambda d: d["start"].__setitem__(slice(None), [0, 1, 0, 1]),     # falling
                   lambda d: d["start"].__setitem__(slice(None), [0, 1, 2, 9]),     # beyond T
                   lambda d: d["c"]["lens"].__setitem__(2, 0)):                     # more than its rows
        st, c, cache, _, _ = append_flags(change)
        assert st == pced.PCED_DEV_BAD_LENGTH
        assert int(c["table"][0, 0]) in changed_blocks(c, cache)  # the first sequence has its token


def test_bad_block_is_not_written(cuda_ok):
    import paper_2601_08670_gb300 as pced
    st, c, cache, x, q = append_flags(lambda d: d["c"]["table"].__setitem__((1, 0), len(d["c"]["k"])))
    assert st == pced.PCED_DEV_BAD_BLOCK
    assert changed_blocks(c, cache) == {int(c["table"][0, 0]), int(c["table"][2, 1])}
    assert torch.equal(q, x[:, :8])  # the queries need no block


def test_length_beyond_the_table_is_flagged(cuda_ok):
    import paper_2601_08670_gb300 as pced
    st, *_ = append_flags(lambda d: d["c"]["lens"].__setitem__(0, 10_000), one=True)
    assert st & pced.PCED_DEV_BAD_LENGTH


def test_position_outside_the_table_is_not_rotated(cuda_ok):
    import paper_2601_08670_gb300 as pced
    st, c, cache, x, q = append_flags(lambda d: d["pos"].__setitem__(slice(None), [0, 8, -1]), rope_rows=8)
    assert st == pced.PCED_DEV_BAD_INDEX
    assert torch.equal(q, x[:, :8])  # (position 0 turns by nothing)


def test_append_beyond_32_bit_offsets(cuda_ok):
    import paper_2601_08670_gb300 as pced
    rng = np.random.default_rng(3)
    Hkv, P, D = 8, 64, 128
    nb = 2 ** 31 // (Hkv * P * D) + 40
    k = torch.empty((nb, Hkv, P, D), dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    summ = torch.zeros((nb, Hkv, 2, D), dtype=torch.int8, device="cuda")
    table = torch.tensor([[nb - 1, nb - 2]], dtype=torch.int32, device="cuda")
    cache = pced.PagedCache(k, v, table, torch.tensor([100], dtype=torch.int32, device="cuda"), summary=summ,
                            key_step=torch.full((Hkv,), 0.03, device="cuda"))
    x = ref.rng_bf16(rng, (100, 32 + 16, D)).cuda()
    start = torch.tensor([0, 100], dtype=torch.int32, device="cuda")
    q = pced.kv_append(cache, x[:, :32], x[:, 32:40], x[:, 40:], tok_start=start)
    first = summ.clone()
    summ.zero_()
    pced.block_summaries(cache)
    torch.cuda.synchronize()
    assert torch.equal(q, x[:, :32])
    assert torch.equal(k[nb - 1], x[:64, 32:40].transpose(0, 1)) and torch.equal(
        v[nb - 2, :, :36], x[64:, 40:].transpose(0, 1))
    assert torch.equal(first, summ) and summ[nb - 2].any()


@pytest.mark.parametrize("Hkv,D", [(2, 64), (8, 128), (3, 128)])
@pytest.mark.parametrize("P", [16, 48, 64, 256])
def test_summaries_of_a_cache(cuda_ok, Hkv, D, P):
    import paper_2601_08670_gb300 as pced
    rng = np.random.default_rng([Hkv, P])
    c = ref.make_cache(rng, [0, 1, P - 1, P, P + 1, 700, 3 * P], Hkv, D, P)
    c["k"][c["table"][5, 0], 0, 3, 5] = float("nan")
    c["k"][c["table"][5, 0], 0, 4, 6] = float("inf")
    c["k"][c["table"][5, 0], 0, 5, 7] = float("-inf")
    old = rng.integers(-127, 128, size=(len(c["k"]), Hkv, 2, D)).astype(np.int8)
    cache = ref.to_device(c, old)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = pced.block_summaries(cache, status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    assert np.array_equal(got.cpu().numpy(), ref.summaries(c, old))


def test_summaries_flag_bad_blocks(cuda_ok):
    import paper_2601_08670_gb300 as pced
    rng = np.random.default_rng(4)
    c = ref.make_cache(rng, [100, 100], 2, 64, 64)
    old = np.zeros((len(c["k"]), 2, 2, 64), np.int8)
    good = c["table"].copy()
    c["table"][0, 1] = -1
    cache = ref.to_device(c, old)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = pced.block_summaries(cache, status=status).cpu().numpy()
    assert int(status.item()) == pced.PCED_DEV_BAD_BLOCK
    want = ref.summaries(dict(c, table=good), old)
    want[good[0, 1]] = 0
    assert np.array_equal(got, want)


@pytest.mark.parametrize("heads", [(4, 2, 64), (8, 1, 128), (28, 4, 128)])
@pytest.mark.parametrize("P", [128, 256, 512])
def test_items_shared_by_clusters(cuda_ok, heads, P):
    # few sequences of many tokens in large pages: several CTAs bring a page's summary together
    run([780, 700, 3 * P], [780, 650, 3 * P - 1], heads, P)
    run([2 * P + 1], [2 * P], heads, P, packed=False)
