"""sample at temperatures beyond the range that counts."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def run(x, u, **kw):
    import paper_2601_08670_gb300 as pced
    logprob = torch.empty(len(x), device="cuda")
    kw = {n: torch.as_tensor(np.asarray(a, np.float32)).cuda() for n, a in kw.items()}
    token = pced.sample(x, torch.as_tensor(np.asarray(u, np.float32)).cuda(), logprob=logprob, **kw)
    return token.cpu().numpy(), logprob.double().cpu().numpy()


def test_temperatures_count_as_1e_37_at_least(cuda_ok):
    # (logits of its size; the log-probability is that of the same temperature)
    x = torch.tensor([[0.0, -2e-38, -5e-38]] * 4, device="cuda")
    t = np.array([1e-40, 1e-38, 1e-37, 1e-45])
    z = np.float32([0.0, -2e-38, -5e-38]).astype(np.float64) / np.float64(np.float32(1e-37))
    w = np.exp(z)
    sums = np.cumsum(w) / w.sum()
    for i in range(3):
        u = (sums[i] + (sums[i - 1] if i else 0)) / 2
        token, lp = run(x, np.full(4, u), temperature=t)
        assert (token == i).all()
        # (the logits' own last bits, 2^-149 of 1e-37: 2^-26; fp32's rounding of a number below 4)
        assert np.abs(lp - np.log(w[i] / w.sum())).max() < 2.0 ** -21
    token, _ = run(x, np.ones(4), temperature=t, min_p=np.full(4, 0.7))  # weights 1, 0.82, 0.61
    assert (token == 1).all()


def test_temperatures_count_as_1e30_at_most(cuda_ok):
    x = torch.tensor([[0.0, -5e29, -1e30]] * 3, device="cuda")  # weights 1, 0.61, 0.37
    t = np.array([1e30, 1e35, np.inf])
    w = np.exp(np.float32([0.0, -5e29, -1e30]).astype(np.float64) / np.float64(np.float32(1e30)))
    for i, low in ((2, 0.0), (2, 0.3), (1, 0.5), (0, 0.9), (0, 1.0)):  # u = 1: the last token kept
        token, lp = run(x, np.ones(3), temperature=t, min_p=np.full(3, low))
        assert (token == i).all(), low
        kept = w[w >= low]
        assert len(kept) == i + 1 and np.abs(lp - np.log(w[i] / kept.sum())).max() < 2.0 ** -21
