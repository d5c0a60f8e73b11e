"""kv_append with starts or lengths that do not fit: exactly the promised tokens are appended, and nothing else in the
pages, the summaries or the rotated queries changes."""
import numpy as np
import pytest
import torch

import paged_ref as ref

pytestmark = pytest.mark.gpu

HQ, HKV, D = 8, 2, 64


def check(lens, T, start, accepted, P=64, cap=None, status=None, one=False):
    """Appends T tokens and compares everything with the tokens of the `accepted` sequences appended alone.

    cap: max_blocks of the table (as make_cache lays it out without)."""
    import paper_2601_08670_gb300 as pced
    rng = np.random.default_rng([len(lens), T, P])
    held = np.minimum(np.maximum(lens, 0), cap * P) if cap else np.asarray(lens)
    c = ref.make_cache(rng, [int(n) for n in held], HKV, D, P, spoil=False)
    if cap:
        c["table"] = c["table"][:, :cap].copy()
    c["lens"] = np.asarray(lens, np.int32)
    summ = rng.integers(-60, 61, size=(len(c["k"]), HKV, 2, D)).astype(np.int8)
    cache = ref.to_device(c, summ)
    x = ref.rng_bf16(rng, (T, HQ + 2 * HKV, D))
    dev = x.cuda()
    q_out = torch.full((T, HQ, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    pced.kv_append(cache, dev[:, :HQ], dev[:, HQ:HQ + HKV], dev[:, HQ + HKV:], q_out=q_out, status=st,
                   tok_start=None if one else torch.tensor(start, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert int(st.item()) == (pced.PCED_DEV_BAD_LENGTH if status is None else status)
    k, v, want, taken = c["k"].clone(), c["v"].clone(), summ.copy(), set()
    for s in accepted:
        t0, t1 = (s, s + 1) if one else (start[s], start[s + 1])
        row = np.arange(lens[s] - (t1 - t0), lens[s])
        b = c["table"][s, row // P]
        k[b, :, row % P] = x[t0:t1, HQ:HQ + HKV]
        v[b, :, row % P] = x[t0:t1, HQ + HKV:]
        taken |= set(range(t0, t1))
        for blk in np.unique(b):
            keys = x[t0:t1, HQ:HQ + HKV].float().numpy()[b == blk]
            for h in range(HKV):
                new = ref.bounds(keys[:, h], c["key_step"][h])
                old = summ[blk, h]
                want[blk, h] = new if 0 in row[b == blk] % P else np.stack([np.maximum(new[0], old[0]),
                                                                          np.minimum(new[1], old[1])])
    same = lambda a, b: torch.equal(a.cpu().view(torch.int16), b.view(torch.int16))
    assert same(cache.k, k) and same(cache.v, v)
    assert np.array_equal(cache.summary.cpu().numpy(), want)
    mine = sorted(taken)
    assert torch.equal(q_out.cpu()[mine], x[mine, :HQ])
    if not one:
        rest = sorted(set(range(T)) - taken)
        assert bool(torch.isnan(q_out[rest]).all())


@pytest.mark.parametrize("start,accepted", [
    ([0, 1, 2, 9], [0, 1]),      # beyond T: that sequence alone
    ([-1, 1, 2, 3], [1, 2]),     # before the first token: that sequence alone
    ([0, 1, 0, 1], [0]),         # falling: that sequence and those after it
    ([3, 1, 2, 3], []),
    ([0, 2, 1, 3], [0])])
def test_starts_that_do_not_fit(cuda_ok, start, accepted):
    check([5, 20, 70], 3, start, accepted)


def test_more_tokens_than_rows(cuda_ok):
    check([5, 20, 0], 3, [0, 1, 2, 3], [0, 1])
    check([5, 2, 70], 9, [0, 1, 5, 9], [0, 2])


@pytest.mark.parametrize("P", [16, 64])
def test_starts_that_name_tokens_twice(cuda_ok, P):
    # long ranges that together touch far more pages than T tokens can
    T = 2000
    check([T, T, T], T, [0, T, 0, T], [0], P=P)
    check([T] * 9, T, [0, T // 2, T, 0, T, 0, T, 0, T, T], [0, 1], P=P)


def test_a_fall_among_many_sequences(cuda_ok):
    # threads that look at several sequences each
    S, at = 700, 333
    start = list(range(S + 1))
    start[at + 1] = 3
    check([20] * S, S, start, range(at), P=16)


@pytest.mark.parametrize("one", [False, True])
@pytest.mark.parametrize("bad", [193, 10_000, 2 ** 31 - 1])
def test_nothing_is_appended_past_the_table(cuda_ok, one, bad):
    # the last row that the table holds is another token's
    check([bad, 20, 70], 3, [0, 1, 2, 3], [1, 2], cap=3, one=one)


def test_a_full_table_is_no_error(cuda_ok):
    check([192, 20, 70], 3, None, [0, 1, 2], cap=3, one=True, status=0)
    check([192, 20, 70], 9, [0, 4, 8, 9], [0, 1, 2], cap=3, status=0)
