"""paged_attention over 8-bit caches whose values are very large or very small: a power of two in their scales is the same
power of two in the outputs, to the last bit."""
import numpy as np
import pytest
import torch

import cache8_ref as ref8
import paged_ref as ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads", [(8, 2, 64), (16, 2, 128)])
@pytest.mark.parametrize("P", [16, 64])
def test_powers_of_two_in_the_values_scales(cuda_ok, heads, P):
    # Values up to 448 2^-3 2^115 = 2^121: a sum of 130 of them still is an fp32 number.  2^-40: nothing of the sums
    # falls below 2^-126.
    import paper_2601_08670_gb300 as pced
    Hq, Hkv, D = heads
    rng = np.random.default_rng(P)
    lens = [1, 2, 40, 130]
    c = ref8.make_cache(rng, lens, Hkv, D, P, spoil=False)
    c["scale"][:, :, 0] = 2.0 ** -9
    q = ref.rng_bf16(rng, (len(lens), Hq, D), 0.3).cuda()
    cache, lse = ref8.to_device(c), [torch.empty((len(lens), Hq), device="cuda") for _ in range(2)]
    want = pced.paged_attention(cache, q, lse=lse[0])
    ref8.check_attention(c, q, want, lse[0])
    own = cache.scale.clone()
    for e in (115, -40):
        cache.scale.copy_(own)
        cache.scale[:, :, 1] *= 2.0 ** e
        got = pced.paged_attention(cache, q, lse=lse[1])
        assert bool(torch.isfinite(got).all())
        assert torch.equal(got.double(), want.double() * 2.0 ** e) and torch.equal(lse[0], lse[1])
