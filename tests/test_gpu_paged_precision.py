"""paged_attention's promise that probabilities are held to 24 bits and that sums are rounded, not cut off: inputs on
which nothing else is inexact enough to hide it, with bounds that 16-bit probabilities and cut sums miss."""
import math

import numpy as np
import pytest
import torch

HEADS = [(4, 1, 64), (8, 2, 128), (8, 1, 64), (7, 1, 128)]  # up to four query heads per kv-head, and more
# Of o = p v / (1 + p), relative: the score is a whole number, times one rounded constant (two roundings of |x| <= 2.9,
# 2.4e-7 after the exponential), exp2 (two units, 2.4e-7), three products of P's parts joined (2^-23 each, 2.4e-7 in
# all), the sum, its reciprocal and the last product (2^-24 each, 1.8e-7): below 1e-6.
P_BOUND = 1e-6
STEPS = 128  # p = exp(-i / 64)


def bf16(x):
    """fp32 rounded to bf16's eight bits, to nearest even."""
    u = np.asarray(x, np.float32).view(np.uint32)
    return ((u + 0x7FFF + (u >> 16 & 1)) & 0xFFFF0000).astype(np.uint32).view(np.float32)


def test_two_parts_miss_the_bound():
    p = np.exp(-np.arange(STEPS) / 64)
    f = p.astype(np.float32)
    hi = bf16(f)
    lo = bf16(f - hi)
    rest = bf16(f - hi - lo)
    assert np.array_equal(hi.astype(np.float64) + lo + rest, f.astype(np.float64))
    err = np.abs((hi.astype(np.float64) + lo) / (1 + p) / (p / (1 + p)) - 1)
    assert err.max() >= 1.5 * P_BOUND


@pytest.mark.gpu
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("P", [16, 64])
def test_probabilities_keep_24_bits(cuda_ok, heads, P):
    import paper_2601_08670_gb300 as pced
    Hq, Hkv, D = heads
    S = STEPS
    k = torch.zeros((S, Hkv, P, D))
    v = torch.zeros((S, Hkv, P, D))
    # two rows: one that scores 0, whose value is 0, and one that scores -i, whose value is 1
    k[:, :, 1, 3] = -torch.arange(S, dtype=torch.float32)[:, None]
    v[:, :, 1] = 1.0
    q = torch.zeros((S, Hq, D))
    q[:, :, 3] = 1.0
    dev = lambda t: t.to(torch.bfloat16).cuda()
    table = torch.arange(S, dtype=torch.int32, device="cuda")[:, None].contiguous()
    cache = pced.PagedCache(dev(k), dev(v), table, torch.full((S,), 2, dtype=torch.int32, device="cuda"))
    out = pced.paged_attention(cache, dev(q), scale=1 / 64).double().cpu().numpy()
    p = np.exp(-np.arange(S) / 64)[:, None, None]
    assert np.abs(out / (p / (1 + p)) - 1).max() <= P_BOUND


# The mean error, with sign, of an output over many channels: what is rounded to nearest errs in both directions and
# averages out, so that a few common roundings of 2^-24 are left (the last product's, exp2's in part); what is cut off
# errs in one direction with every tile that is added.
TILES = 500  # of a CTA; every other one is a warpgroup's
MEAN_BOUND = 2.0 ** -20


def test_cut_sums_miss_the_bound():
    rng = np.random.default_rng(1)
    add = rng.uniform(10, 24, size=(TILES // 2, 1000)).astype(np.float32)
    cut = np.zeros(1000, np.float32)
    for t in add:
        x = cut.astype(np.float64) + t
        cut = x.astype(np.float32)
        cut = np.where(cut > x, np.nextafter(cut, np.float32(0)), cut)
    err = cut / add.sum(axis=0, dtype=np.float64) - 1
    assert -err.mean() >= 2 * MEAN_BOUND


@pytest.mark.gpu
@pytest.mark.parametrize("G", [4, 8])
def test_sums_of_many_tiles_are_rounded(cuda_ok, G):
    import paper_2601_08670_gb300 as pced
    P, D = 256, 64
    g = torch.Generator(device="cuda").manual_seed(G)
    n = torch.cuda.get_device_properties(0).multi_processor_count * TILES * 64
    nb = n // P
    k = torch.zeros((nb, 1, P, D), dtype=torch.bfloat16, device="cuda")
    k[..., 0] = torch.randint(-64, 1, (nb, 1, P), device="cuda", generator=g).to(torch.bfloat16)
    v = (1 + torch.rand((nb, 1, P, D), device="cuda", generator=g)).to(torch.bfloat16)
    table = torch.randperm(nb, device="cuda", generator=g).to(torch.int32)[None].contiguous()
    cache = pced.PagedCache(k, v, table, torch.tensor([nb * P], dtype=torch.int32, device="cuda"))
    q = torch.zeros((1, G, D), dtype=torch.bfloat16, device="cuda")
    q[0, :, 0] = torch.arange(1, G + 1, device="cuda") / 4
    out = pced.paged_attention(cache, q, scale=1 / 64)[0].double()
    z = k[:, 0, :, 0].reshape(-1).double()
    want = torch.zeros((G, D), dtype=torch.float64, device="cuda")
    total = torch.zeros(G, dtype=torch.float64, device="cuda")
    for i in range(0, nb, 2048):
        p = torch.exp(z[i * P:(i + 2048) * P, None] * q[0, :, 0].double() / 64)
        want += p.T @ v[i:i + 2048, 0].reshape(-1, D).double()
        total += p.sum(0)
    want /= total[:, None]
    mean = (out / want - 1).mean()
    assert abs(float(mean)) <= MEAN_BOUND
