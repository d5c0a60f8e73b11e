"""block_select against the definition in whole numbers: the choice is equal, ties included."""
import numpy as np
import pytest
import torch

import paged_ref as ref

pytestmark = pytest.mark.gpu


def run(lens, heads, P, n_sel, n_first=1, n_last=1, seed=0, coarse=0, change=None, status=0):
    import paper_2601_08670_gb300 as pced
    Hq, Hkv, D = heads
    rng = np.random.default_rng([seed, Hq, P, n_sel])
    table, nb = ref.make_table(rng, lens, P)
    c = dict(table=table, lens=np.asarray(lens, np.int32), P=P, Hkv=Hkv, D=D)
    summ = rng.integers(-127, 128, size=(nb, Hkv, 2, D)).astype(np.int8)
    if coarse:  # few different blocks: many ties
        summ = summ[rng.integers(0, coarse, size=nb)].copy()
    q = ref.rng_bf16(rng, (len(lens), Hq, D))
    if change:
        change(c, summ, q)
    t = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    cache = pced.PagedCache(None, None, t(c["table"]), t(c["lens"]), block_rows=P, summary=t(summ))
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    sel = pced.block_select(cache, q.cuda(), n_sel, n_first, n_last, status=st)
    torch.cuda.synchronize()
    assert int(st.item()) == status
    assert np.array_equal(sel.cpu().numpy(), ref.select(c, summ, q, n_sel, n_first, n_last))


HEADS = [(8, 2, 64), (16, 2, 64), (28, 4, 128), (32, 8, 128), (3, 3, 64)]


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("n_sel,n_first,n_last", [(1, 0, 0), (2, 1, 1), (7, 0, 3), (33, 2, 0), (300, 1, 1)])
def test_choices(cuda_ok, heads, n_sel, n_first, n_last):
    P = 16
    run([0, 1, 16, 17, 100, 33 * 16, 34 * 16 - 1, 5000], heads, P, n_sel, n_first, n_last)


@pytest.mark.parametrize("P", [16, 64, 192])
def test_ties_go_to_the_lowest_block(cuda_ok, P):
    run([40 * P, 257 * P + 1, 300 * P], (8, 2, 64), P, 20, coarse=3)
    run([40 * P, 257 * P + 1, 300 * P], (8, 2, 64), P, 21, 0, 0, coarse=1)  # all blocks alike


@pytest.mark.parametrize("blocks", [255, 256, 257, 2048, 2049, 8191, 20_000, 32_000])
def test_long_rows(cuda_ok, blocks):
    run([blocks * 16, blocks * 16 - 15, 16 * 40], (4, 1, 128), 16, 64, seed=blocks)


def test_many_sequences(cuda_ok):
    run(list(range(0, 1000, 2)), (8, 2, 64), 16, 9)


def test_queries_of_one_size_or_none(cuda_ok):
    def change(c, summ, q):
        q[0] = 0            # every block scores 0
        q[1, 3] = float("inf")
        q[2, 0, 5] = float("nan")
        q[3] *= 1e-30       # steps are relative to the largest part
    run([1000, 1100, 1200, 1300], (8, 2, 64), 16, 10, change=change)


def test_bad_entries_come_last(cuda_ok):
    import paper_2601_08670_gb300 as pced

    def change(c, summ, q):
        c["table"][0, 3:60] = -1
        c["table"][1, 5] = len(summ)
    run([1000, 1100], (8, 2, 64), 16, 10, change=change, status=pced.PCED_DEV_BAD_BLOCK)


def test_extreme_summaries(cuda_ok):
    # the largest scores the 8-bit numbers allow
    def change(c, summ, q):
        q[:] = 1.0
        summ[:, :, 0] = 127
        summ[:, :, 1] = -127
        q[1] = -1.0
        summ[c["table"][0, 30]] = -127
        summ[c["table"][1, 31], :, 1] = 127
    run([1000, 1100], (16, 2, 64), 16, 40, change=change)


def test_queries_next_to_zero(cuda_ok):
    """127 / m is infinite: all scores are 0, so the lowest blocks follow the first and the last ones."""
    import paper_2601_08670_gb300 as pced
    rng = np.random.default_rng(5)
    for blocks in (40, 700):  # counted, and by the radix
        table, nb = ref.make_table(rng, [blocks * 16], 16)
        summ = torch.from_numpy(rng.integers(-127, 128, size=(nb, 2, 2, 64)).astype(np.int8)).cuda()
        cache = pced.PagedCache(None, None, torch.from_numpy(table).cuda(),
                                torch.tensor([blocks * 16], dtype=torch.int32, device="cuda"), block_rows=16,
                                summary=summ)
        q = (ref.rng_bf16(rng, (1, 8, 64)).float().clamp(-2, 2) * 2.0 ** -126).to(torch.bfloat16).cuda()
        sel = pced.block_select(cache, q, 10, 1, 2).cpu().numpy()
        assert np.array_equal(sel, np.tile([*range(8), blocks - 2, blocks - 1], (1, 2, 1)))
