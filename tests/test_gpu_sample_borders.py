"""sample where an error of 2^-29 in a weight would show: borders of two tokens next to u."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

# A weight is off by at most 2^-30 of itself.  Of a row of two values, where the first half of the tokens holds f of the
# weight, the border of the halves is off by f (1 - f) of that: 2^-32; its sums add less than 2^-38 (sixteen terms below
# 2^-19 each, added in 32 bits, by a weight of 16).
BORDER = 2.0 ** -31.7


def run(x, u):
    import paper_2601_08670_gb300 as pced
    return pced.sample(x, torch.from_numpy(u).cuda()).cpu().numpy()


def halves(d, n):
    """Rows of n tokens of logit d[i] and n of 0, u as near to the border as 32 bits say, and how near: (x, u, token, margin)."""
    w = np.exp(d.astype(np.float64))
    f = w / (1 + w)
    u = f.astype(np.float32)
    x = torch.zeros((len(d), 2 * n), device="cuda")
    x[:, :n] = torch.from_numpy(d)[:, None].cuda()
    return x, u, np.where(u < f, n - 1, n), np.abs(u - f)


@pytest.mark.parametrize("n", [600, 2500])
def test_borders_that_an_error_of_2_to_the_minus_29_moves(cuda_ok, n):
    d = np.array([0xBEA0C44D, 0xBE7F0C35, 0xBED8787D, 0xBE521AD0, 0xBEC1C99C, 0xBED885B8], np.uint32).view(np.float32)
    x, u, want, margin = halves(d, n)
    assert (margin > BORDER).all()
    token = run(x, u)
    assert np.array_equal(token, want)


def test_borders_next_to_u(cuda_ok):
    rng = np.random.default_rng(1)
    d = -rng.uniform(0.01, 0.9, 200_000).astype(np.float32)
    near = halves(d, 0)[3]
    d = d[(near > BORDER) & (near < 2.0 ** -29)]
    assert len(d) > 2000
    for at in range(0, len(d), 2000):
        x, u, want, _ = halves(d[at:at + 2000], 600)
        token = run(x, u)
        assert np.array_equal(token, want)
