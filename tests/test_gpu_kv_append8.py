"""kv_append into 8-bit caches against its definition, byte for byte: scales, moved rows, rotation, summaries, and what stays
untouched."""
import numpy as np
import pytest
import torch

import cache8_ref as ref8
import paged_ref as ref

pytestmark = pytest.mark.gpu


def same_numbers(got, want):
    """Bytes that stand for the same numbers (0x7F and 0xFF are both not a number)."""
    got, want = got.copy(), want.copy()
    got[(got & 0x7F) == ref8.NAN] = ref8.NAN
    want[(want & 0x7F) == ref8.NAN] = ref8.NAN
    return np.array_equal(got, want)


def run(lens, new, heads, P, rope=True, positions=None, one=False, spare=5, seed=0, q_none=False, summary=True, sigma=1.5,
        change=None, packed=True):
    import paper_2601_08670_gb300 as pced
    Hq, Hkv, D = heads
    rng = np.random.default_rng([seed, Hq, P, len(lens)])
    c = ref8.make_cache(rng, lens, Hkv, D, P, spare=spare, spoil=False)
    summ = rng.integers(-60, 61, size=(len(c["k"]), Hkv, 2, D)).astype(np.int8) if summary else None
    T = sum(new)
    # rows far larger and far smaller than their block's scale
    qkv = ref.rng_bf16(rng, (T, Hq + 2 * Hkv, D), sigma) * torch.from_numpy(np.exp2(rng.integers(-9, 4, size=(T, 1, 1)))).to(
        torch.bfloat16)
    if change is not None:
        change(c, qkv)
    cache = ref8.to_device(c, summ)
    dev = qkv.cuda()
    q, k, v = dev[:, :Hq], dev[:, Hq:Hq + Hkv], dev[:, Hq + Hkv:]
    if not packed:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    row = np.concatenate([np.arange(n - m, n) for n, m in zip(lens, new)]).astype(np.int64)
    pos = row if positions is None else positions
    tab = pced.rope_table(1e4, D, int(pos.max()) + 1) if rope else None
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    q_out = pced.kv_append(cache, None if q_none else q, k, v, rope=tab,
                           tok_start=None if one else torch.from_numpy(start).cuda(),
                           positions=None if positions is None else torch.from_numpy(pos.astype(np.int32)).cuda(),
                           status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    x = qkv.float().numpy()
    rot = x[:, :Hq + Hkv]
    if rope:
        rot = ref8.rotated32(rot, tab.cpu().numpy()[pos])
    if q_none:
        assert q_out is None
    else:
        want = torch.from_numpy(rot[:, :Hq].copy()).to(torch.bfloat16)
        assert np.array_equal(q_out.float().cpu().numpy(), want.float().numpy(), equal_nan=True)
    want, want_summ = ref8.append(c, rot[:, Hq:], x[:, Hq + Hkv:], new, summ)
    assert np.array_equal(cache.scale.cpu().numpy(), want["scale"])
    for name in ("k", "v"):
        assert same_numbers(getattr(cache, name).view(torch.uint8).cpu().numpy(), want[name]), name
    if summary:
        assert np.array_equal(cache.summary.cpu().numpy(), want_summ)


HEADS = [(8, 2, 64), (16, 2, 64), (28, 4, 128), (32, 8, 128), (3, 3, 64)]


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("P", [16, 64, 192])
def test_one_token_per_sequence(cuda_ok, heads, P):
    lens = [1, 2, 16, 17, 64, 65, 192, 193, 700]
    run(lens, [1] * len(lens), heads, P, one=True)
    run(lens, [1] * len(lens), heads, P, one=False, rope=False, summary=False)


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("P", [16, 64, 256])
def test_ragged_prompts(cuda_ok, heads, P):
    # whole sequences, parts that begin and end inside blocks, sequences without tokens
    lens = [0, 1, 63, 64, 65, 300, 129, 40, 500]
    new = [0, 1, 63, 64, 65, 300, 100, 0, 7]
    run(lens, new, heads, P, packed=P != 64)


@pytest.mark.parametrize("seed", range(4))
def test_every_move(cuda_ok, seed):
    # few new rows in blocks that hold many: by one token, by several, by several kv-heads a CTA
    run([250] * 40, [1] * 40, (8, 2, 64), 256, one=True, seed=seed)
    run([250] * 40, [2] * 40, (32, 8, 128), 256, seed=seed)
    run([260] * 8, [10] * 8, (28, 4, 128), 256, seed=seed)


def test_many_sequences_and_one_long_prompt(cuda_ok):
    run([5] * 700, [2] * 700, (8, 2, 64), 16)
    run([3000], [2900], (8, 2, 64), 256, packed=False)


def test_positions_of_their_own(cuda_ok):
    run([10, 20, 30], [3, 20, 1], (8, 2, 64), 16, positions=np.arange(24) * 37 % 101)


def test_keys_without_queries(cuda_ok):
    run([10, 20, 30], [3, 20, 1], (2, 2, 64), 16, q_none=True)
    run([10, 20, 30], [1, 1, 1], (2, 2, 128), 16, q_none=True, one=True)


@pytest.mark.parametrize("one", [True, False])
def test_zeros_infinities_and_what_is_no_number(cuda_ok, one):
    def change(c, qkv):
        qkv[0] = 0.0
        qkv[1, :, 3], qkv[1, :, 9] = float("inf"), float("-inf")
        qkv[2, :, 5] = float("nan")
        qkv[3] = float("nan")
        qkv[4] *= 2.0 ** 120       # the largest scales
        qkv[5] *= 2.0 ** -120      # below the smallest one
    for lens in ([1] * 6, [17] * 6, [7] * 6):
        run(lens, [1] * 6, (8, 2, 64), 16, one=one, rope=False, change=change)


@pytest.mark.parametrize("one", [True, False])
def test_scales_that_no_append_wrote(cuda_ok, one):
    # any scale above 0, one that was never written, one that is not a number: those count as none
    def change(c, qkv):
        for s, x in enumerate((0.013, 0.0, float("nan"), 3e-5)):
            c["scale"][c["table"][s, 0]] = x
    run([7] * 4, [1] * 4, (8, 2, 64), 16, one=one, change=change)


def test_a_block_filled_row_by_row_and_at_once(cuda_ok):
    # the same scale; a row can be off by what moved below the smallest numbers, half a step of the last scale: 2^-10
    import paper_2601_08670_gb300 as pced
    rng = np.random.default_rng(3)
    P, n = 64, 200
    c = ref8.make_cache(rng, [n], 2, 64, P, spoil=False)
    x = (ref.rng_bf16(rng, (n, 12, 64)).float() * torch.from_numpy(np.exp2(rng.integers(-12, 5, size=(n, 1, 1))))).to(
        torch.bfloat16).cuda()
    at_once, by_row = ref8.to_device(c), ref8.to_device(c)
    start = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    pced.kv_append(at_once, x[:, :8], x[:, 8:10], x[:, 10:], tok_start=start)
    for i in range(n):
        by_row.seq_len.fill_(i + 1)
        pced.kv_append(by_row, x[i:i + 1, :8], x[i:i + 1, 8:10], x[i:i + 1, 10:])
    assert torch.equal(at_once.scale, by_row.scale)
    scale = at_once.scale.double()
    for i, name in enumerate(("k", "v")):
        a, b = (ref8.numbers(getattr(t, name).view(torch.uint8).cpu().numpy()) for t in (at_once, by_row))
        used = c["table"][0, :(n + P - 1) // P]
        assert np.abs(a - b)[used].max() <= 2.0 ** -9  # (a row's own rounding, then the move's)
        assert (a != b)[used].mean() < 0.05
    assert bool((scale > 0).all())


def test_nothing_else_is_touched(cuda_ok):
    import paper_2601_08670_gb300 as pced
    rng = np.random.default_rng(1)
    lens = [5, 0, 70]
    c = ref8.make_cache(rng, lens, 2, 64, 64, spoil=False)
    cache = ref8.to_device(c, np.zeros((len(c["k"]), 2, 2, 64), np.int8))
    x = ref.rng_bf16(rng, (3, 12, 64)).cuda()
    q_out = torch.full((3, 8, 64), float("nan"), dtype=torch.bfloat16, device="cuda")
    pced.kv_append(cache, x[:, :8], x[:, 8:10], x[:, 10:], q_out=q_out)
    torch.cuda.synchronize()
    assert torch.equal(q_out[[0, 2]], x[[0, 2], :8]) and not q_out[1].any()
    b = c["table"][1, 0]  # the idle sequence's
    assert np.array_equal(cache.k[b].view(torch.uint8).cpu().numpy(), c["k"][b]) and not cache.summary[int(b)].any()
    assert np.array_equal(cache.scale[b].cpu().numpy(), c["scale"][b])


def test_bad_lengths_blocks_and_starts(cuda_ok):
    import paper_2601_08670_gb300 as pced
    rng = np.random.default_rng(2)
    for lens, table, start, bit in ([[200, 3], {}, None, pced.PCED_DEV_BAD_LENGTH], [[-1, 3], {}, None, pced.PCED_DEV_BAD_LENGTH],
                                    [[40, 3], {(0, 0): 99}, None, pced.PCED_DEV_BAD_BLOCK],
                                    [[40, 3], {(0, 0): -7}, [0, 1, 2], pced.PCED_DEV_BAD_BLOCK],
                                    [[40, 3], {}, [0, -1, 2], pced.PCED_DEV_BAD_LENGTH],
                                    [[0, 3], {}, [0, 1, 2], pced.PCED_DEV_BAD_LENGTH],
                                    [[40, 3], {}, [0, 5, 2], pced.PCED_DEV_BAD_LENGTH]):
        c = ref8.make_cache(rng, [40, 3], 2, 64, 64, spoil=False)
        c["table"] = c["table"][:, :1].copy()
        for at, b in table.items():
            c["table"][at] = b
        c["lens"] = np.array(lens, np.int32)
        cache = ref8.to_device(c)
        x = ref.rng_bf16(rng, (2, 12, 64), 30.0).cuda()
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        pced.kv_append(cache, x[:, :8], x[:, 8:10], x[:, 10:], status=status,
                       tok_start=None if start is None else torch.tensor(start, dtype=torch.int32, device="cuda"))
        assert int(status.item()) == bit
        # the other sequence has its row (but where the starts fall before it), and all else is as it was
        got = cache.k.view(torch.uint8).cpu().numpy()
        changed = sorted(set(np.nonzero((got != c["k"]).any(axis=(1, 2, 3)))[0].tolist()))
        assert changed in ([], [int(c["table"][1, 0])]), (lens, table, start, changed)
        if start is None:
            assert changed
