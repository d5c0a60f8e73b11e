"""sample against its definition in 64 bits: sizes, types, ties, masks, every cut, parameters at their ends, strides, and
that it depends on nothing else."""
import numpy as np
import pytest
import torch

import sample_ref as ref

pytestmark = pytest.mark.gpu

# A weight is off by at most 2^-31 of itself (the table and the series, half a step of 2^-31 each; the series' own error
# 2^-31; an argument off by 2^-31), sixteen of them together by a step of 2^-42 more; so are sums of them.  Where u (or p)
# lies nearer than twice that to a border of two tokens, the neighbour is as right.
MARGIN = 2.0 ** -30
# logprob: fp32's rounding of a number below 32 (2^-20), and what the sum is off
LOGPROB = 2.0 ** -19


def run(x, u, t=None, k=None, p=None, low=None, status=0, **kw):
    """(tokens, logprobs) with every parameter an array or None; x: a device tensor [rows, V]."""
    import paper_2601_08670_gb300 as pced
    dev = lambda a, d: None if a is None else torch.as_tensor(np.asarray(a, d)).cuda()
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    logprob = torch.full((len(x),), float("nan"), device="cuda")
    tok = pced.sample(x, dev(u, np.float32), temperature=dev(t, np.float32), top_k=dev(k, np.int32), top_p=dev(p, np.float32),
                      min_p=dev(low, np.float32), logprob=logprob, status=word, **kw)
    torch.cuda.synchronize()
    assert int(word.item()) == status
    return tok.cpu().numpy(), logprob.cpu().numpy()


def check(x, u, t=None, k=None, p=None, low=None, near=0, **kw):
    """near: rows that may lie too near a border to say."""
    tok, lp = run(x, u, t, k, p, low, **kw)
    h = x.double().cpu().numpy()
    n = len(h)
    args = [np.asarray(a if a is not None else np.full(n, d, np.float32), np.float32).astype(np.float64)
            for a, d in ((u, 0), (t, 1), (p, 1), (low, 0))]
    left = near
    for i in range(n):
        want, want_lp, margin = ref.row(h[i], args[0][i], args[1][i], 0 if k is None else int(k[i]), args[2][i], args[3][i])
        if margin < MARGIN and tok[i] != want:
            left -= 1
            continue
        assert tok[i] == want, (i, tok[i], want, margin)
        assert lp[i] == want_lp or abs(lp[i] - want_lp) <= LOGPROB * max(1.0, abs(want_lp)), (i, lp[i], want_lp)
    assert left >= 0


def logits(rows, V, seed, bf16=False, sigma=2.5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.empty((rows, V), device="cuda").normal_(0, sigma, generator=g)
    return x.to(torch.bfloat16) if bf16 else x


def numbers(rows, seed):
    return (np.random.default_rng(seed).integers(0, 1 << 24, rows) + 0.5) * 2.0 ** -24


def mixed(rows, seed):
    r = np.random.default_rng([seed, 1])
    return dict(t=r.choice([0.0, 0.3, 0.7, 1.0, 1.6, 5.0], rows), k=r.choice([-1, 0, 1, 2, 7, 50, 700, 10 ** 6], rows),
                p=r.choice([0.0, 0.1, 0.5, 0.9, 0.99, 0.9999, 1.0, 2.0], rows),
                low=r.choice([-1.0, 0.0, 0.001, 0.05, 0.5, 1.0, 3.0], rows))


SIZES = [1, 2, 3, 7, 8, 31, 33, 255, 256, 257, 1000, 2047, 2049, 4099, 16_385, 50_257, 151_936]


@pytest.mark.parametrize("V", SIZES)
@pytest.mark.parametrize("bf16", [False, True])
def test_mixed_requests(cuda_ok, V, bf16):
    rows = 40
    check(logits(rows, V, V, bf16), numbers(rows, V), **mixed(rows, V))


@pytest.mark.parametrize("cut", ["none", "k", "p", "kp", "low", "all"])
@pytest.mark.parametrize("rows,V", [(1, 128_256), (3, 32_000), (80, 128_256), (600, 5000)])
def test_each_cut(cuda_ok, cut, rows, V):
    r = np.random.default_rng([rows, V, 2])
    kw = dict(t=r.uniform(0.3, 1.5, rows))
    if cut in ("k", "kp", "all"):
        kw["k"] = r.integers(2, V // 2, rows)
    if cut in ("p", "kp", "all"):
        kw["p"] = r.uniform(0.05, 0.9999, rows)
    if cut in ("low", "all"):
        kw["low"] = 10.0 ** r.uniform(-5, 0, rows)
    check(logits(rows, V, rows + V), numbers(rows, rows), **kw)


@pytest.mark.parametrize("V", [300_001, 393_216])
@pytest.mark.parametrize("bf16", [False, True])
def test_the_largest_vocabularies(cuda_ok, V, bf16):
    check(logits(5, V, 3, bf16), numbers(5, 3), t=np.full(5, 1.2), k=[0, 90_000, 5, 0, 0], p=[1, 0.99, 0.5, 0.9, 1],
          low=[0, 0, 0, 0, 1e-3])


@pytest.mark.parametrize("rows", [10, 19, 38, 64, 120, 160])
@pytest.mark.parametrize("V", [9000, 70_001])
def test_rows_split_over_any_number_of_ctas(cuda_ok, rows, V):
    check(logits(rows, V, rows, rows % 3 == 1), numbers(rows, V), near=1, **mixed(rows, rows + V))


def test_every_border_of_a_few_tokens(cuda_ok):
    # u just below and just above each border: whole numbers as weights, so that the borders are known
    w = np.array([3, 1, 4, 1, 5, 9, 2, 6], np.float64)
    edge = np.cumsum(w) / w.sum()
    u = np.concatenate([[0.0], edge[:-1] - 2.0 ** -20, edge[:-1] + 2.0 ** -20, [1.0]]).astype(np.float32)
    want = np.concatenate([[0], np.arange(7), np.arange(1, 8), [7]])
    x = torch.from_numpy(np.log(w).astype(np.float32)).cuda().expand(len(u), -1)
    tok, _ = run(x.contiguous(), u)
    assert np.array_equal(tok, want)


@pytest.mark.parametrize("bf16", [False, True])
def test_ties_everywhere(cuda_ok, bf16):
    # a handful of values over all tokens: cuts fall inside ties, which the lower tokens win
    rows, V = 60, 20_000
    g = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randint(0, 4, (rows, V), device="cuda", generator=g).float()
    x[:5] = 1.0   # nothing but ties
    x[5:8] = -0.0
    x[6, 100:] = 0.0
    r = np.random.default_rng(4)
    check(x.to(torch.bfloat16) if bf16 else x, numbers(rows, 4), t=r.choice([0.5, 1.0, 100.0], rows),
          k=r.choice([0, 2, 513, 6000, 15_000], rows), p=r.choice([1.0, 0.001, 0.3, 0.77], rows))


def test_ties_that_end_at_a_token(cuda_ok):
    # of equal logits a cut keeps the first: with u = 1 the last kept token shows where
    V = 30_000
    x = torch.zeros((6, V), device="cuda")
    k = np.array([2, 511, 512, 513, 1025, 29_999], np.int32)
    tok, lp = run(x, np.ones(6), k=k)
    assert np.array_equal(tok, k - 1) and np.allclose(lp, -np.log(k), rtol=2.0 ** -20)
    p = np.array([1, 5, 1000, 20_000, 29_999, 30_000]) / V - 1e-6
    tok, _ = run(x, np.ones(6), p=p)
    assert np.array_equal(tok, np.ceil(p.astype(np.float32).astype(np.float64) * V) - 1)


def test_masked_tokens_are_never_drawn(cuda_ok):
    rows, V = 64, 40_000
    x = logits(rows, V, 5)
    g = torch.Generator(device="cuda").manual_seed(5)
    off = torch.rand((rows, V), device="cuda", generator=g) < 0.99
    off[:, 17] = False
    off[3] = True
    off[3, 39_999] = False  # one token left
    off[4] = True           # none
    x = x.masked_fill(off, float("-inf"))
    x[7, ::2] = float("nan")
    kw = mixed(rows, 5)
    check(x, numbers(rows, 5), **kw)
    tok, lp = run(x, numbers(rows, 5), **kw)
    assert tok[3] == 39_999 and tok[4] == -1 and np.isneginf(lp[4])


def test_infinite_and_very_large_logits(cuda_ok):
    x = logits(8, 3000, 6)
    x[0, [5, 900, 2000]] = float("inf")
    x[1] *= 1e36
    x[2] = 3e38
    x[3] = -3e38
    x[4, :] = float("-inf")
    x[5] *= 1e-40
    x[6, 1:] = -1e30
    for kw in (dict(), dict(k=np.full(8, 2)), dict(p=np.full(8, 0.4)), dict(low=np.full(8, 0.1)),
               dict(t=np.full(8, 1e-6)), dict(t=np.full(8, 1e20))):
        check(x, numbers(8, 6), **kw)
    tok, lp = run(x[:1], [0.5])
    assert tok[0] == 900 and abs(lp[0] + np.log(3)) < 1e-6


@pytest.mark.parametrize("t", [1e-38, 1e-6, 0.01, 30.0, 1e6, 1e29, 1e31, float("inf")])
def test_temperatures_of_any_size(cuda_ok, t):
    rows, V = 12, 9000
    r = np.random.default_rng(7)
    check(logits(rows, V, 7), numbers(rows, 7), t=np.full(rows, t), k=r.choice([0, 100, 4000], rows),
          p=r.choice([1.0, 0.2, 0.9], rows))


def test_parameters_out_of_range(cuda_ok):
    import paper_2601_08670_gb300 as pced
    nan = float("nan")
    x = logits(9, 500, 8)
    ok = dict(t=np.ones(9), p=np.full(9, 0.9), low=np.full(9, 0.01), k=np.full(9, 50))
    u = numbers(9, 8)
    good, _ = run(x, u, **ok)
    for name, i, v in (("t", 0, -1.0), ("t", 1, nan), ("p", 2, nan), ("low", 3, nan), ("u", 4, -0.1), ("u", 5, 1.5),
                       ("u", 6, nan)):
        kw, uu = {a: b.copy() for a, b in ok.items()}, u.copy()
        (uu if name == "u" else kw[name])[i] = v
        tok, lp = run(x, uu, status=pced.PCED_DEV_BAD_PARAM, **kw)
        assert tok[i] == -1 and np.isneginf(lp[i])
        assert np.array_equal(np.delete(tok, i), np.delete(good, i))


def test_strided_rows_of_any_alignment(cuda_ok):
    for dtype in (torch.float32, torch.bfloat16):
        big = logits(6, 5011, 9).to(dtype)
        for first in range(9):
            x = big[:, first:first + 4097]
            assert not x.is_contiguous()
            check(x, numbers(6, first), t=np.full(6, 0.8), k=[0, 3, 600, 0, 0, 1], p=[1, 1, 0.9, 0.5, 1, 1],
                  low=[0, 0, 0, 0, 0.02, 0])


def test_frequencies(cuda_ok):
    # u on a grid of 20,000: every token as often as its weight says, but for one
    n = 20_000
    w = np.random.default_rng(10).uniform(0.1, 1, 40)
    x = torch.from_numpy(np.log(w).astype(np.float32)).cuda().expand(n, -1).contiguous()
    tok, lp = run(x, (np.arange(n) + 0.5) / n)
    share = w / w.sum()
    assert np.abs(np.bincount(tok, minlength=40) - n * share).max() <= 1.0 + n * 40 * 2.0 ** -23
    assert np.allclose(lp, np.log(share)[tok], atol=2.0 ** -19)


def test_the_same_again_and_beside_other_rows(cuda_ok):
    # a row's token does not depend on the rows beside it, which decide how many CTAs share it
    V = 50_000
    x = logits(400, V, 11)
    u = numbers(400, 11)
    kw = mixed(400, 11)
    all_, lp = run(x, u, **kw)
    again, lp2 = run(x, u, **kw)
    assert np.array_equal(all_, again) and np.array_equal(lp, lp2)
    for a, b in ((0, 1), (7, 9), (100, 140)):
        tok, lp3 = run(x[a:b], u[a:b], **{n: v[a:b] for n, v in kw.items()})
        assert np.array_equal(tok, all_[a:b]) and np.array_equal(lp3, lp[a:b])


def test_inputs_stay_as_they_are(cuda_ok):
    x = logits(4, 1001, 12)
    before = x.clone()
    run(x, numbers(4, 12), p=np.full(4, 0.5))
    assert torch.equal(x, before)


def test_no_rows(cuda_ok):
    tok, _ = run(torch.empty((0, 10), device="cuda"), np.zeros(0))
    assert tok.shape == (0,)


def test_another_stream_and_graph_replays(cuda_ok):
    import paper_2601_08670_gb300 as pced
    x, u = logits(5, 20_000, 13), torch.rand(5, device="cuda")
    p = torch.full((5,), 0.8, device="cuda")
    want = pced.sample(x, u, top_p=p).cpu()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = pced.sample(x, u, top_p=p, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got.cpu(), want)
    g, out = torch.cuda.CUDAGraph(), torch.empty(5, dtype=torch.int32, device="cuda")
    with torch.cuda.graph(g):
        pced.sample(x, u, top_p=p, token=out)
    for _ in range(3):  # the same graph with other random numbers and logits in place
        x.normal_(0, 3)
        u.uniform_()
        want = pced.sample(x, u, top_p=p).cpu()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.cpu(), want)


@pytest.mark.parametrize("V,rows", [(151936, 160), (250001, 170), (300001, 153)])
def test_one_value_almost_everywhere(cuda_ok, V, rows):
    # a CTA's share of a row in one range, of weights with any low bits; p ends inside it
    x = torch.zeros((rows, V), dtype=torch.bfloat16, device="cuda")
    x[:, ::1000] = 1.0
    t = np.linspace(0.31, 1.7, rows).astype(np.float32)
    share = np.linspace(0.05, 0.97, rows).astype(np.float32)
    u = numbers(rows, 4)
    tok, lp = run(x, u, t=t, p=share)
    for i in range(rows):
        # (all ones first, then so many zeros that the share is reached)
        ones, w = (V + 999) // 1000, np.exp(-1 / np.float64(t[i]))
        all_ = ones + (V - ones) * w
        want = np.float64(share[i]) * all_
        zeros = max(0, int(np.ceil((want - ones) / w)))
        if min(abs((want - ones) / w - z) for z in (zeros, zeros - 1)) * w < MARGIN * all_ or want < ones:
            continue
        # the kept zeros are the first ones; a thousand tokens are a one and 999 zeros
        last = zeros + (zeros - 1) // 999 + 1 if zeros else 0  # tokens up to the last kept zero
        total = ones + zeros * w
        goal = np.float64(np.float32(u[i])) * total
        order = np.arange(V)
        kept = (order % 1000 == 0) | (order < last)
        assert int(((order % 1000 != 0) & kept).sum()) == zeros
        sums = np.cumsum(np.where(order % 1000 == 0, 1.0, w) * kept)
        at = int(np.searchsorted(sums, goal, side="right"))
        if np.abs(sums - goal).min() < MARGIN * total:
            continue
        assert tok[i] == at, i
        want_lp = np.log((1.0 if at % 1000 == 0 else w) / total)
        assert abs(lp[i] - want_lp) <= LOGPROB * max(1.0, abs(want_lp))


@pytest.mark.parametrize("u", [0.0, 1.0])
@pytest.mark.parametrize("k", [0, 5, 50, 3000])
def test_the_smallest_weights_beside_a_large_one(cuda_ok, u, k):
    # weights of 2^-45 of the largest, at the ends of the order: some token is drawn, and one that is kept
    for V in (600, 5000, 128256):
        x = torch.zeros((3, V), device="cuda")
        x[:, V // 2] = 45 * float(np.log(2))
        x[1, :V // 4] = -float("inf")
        x[2] += torch.linspace(-1e-3, 1e-3, V, device="cuda")
        tok, lp = run(x, np.full(3, u), k=None if k == 0 else np.full(3, k))
        h = x.cpu().numpy()
        for i in range(3):
            assert 0 <= tok[i] < V and np.isfinite(h[i, tok[i]]) and np.isfinite(lp[i])
            if 0 < k < V:
                assert tok[i] in ref.order(h[i].astype(np.float64))[:k]
