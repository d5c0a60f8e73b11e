"""The example's loop processes logits, and normalises what comes of it before experts are compared: its log-probabilities
and choices against the same in plain 64-bit arithmetic."""
import os
import sys

import numpy as np
import pytest
import torch

import paged_ref as ref

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))

B, N, V = 2, 2, 1000
GAMMA, BETA = 2.5, 0.5


def choice(lp, r):
    """Tokens and experts of Eq. 2 and Eq. 3, and the score's lead over any other (token, expert)."""
    lp = lp.reshape(B, N + 1, V)
    s = (1 + BETA) * lp[:, 1:] - BETA * lp[:, :1] + GAMMA * np.log(r)[:, :, None]
    s = np.where(np.isnan(s), -np.inf, s).reshape(B, -1)
    best = s.argmax(1)
    top2 = np.sort(s, axis=1)[:, -2:]
    return best % V, best // V + 1, top2[:, 1] - top2[:, 0]


@pytest.mark.parametrize("masked,rep", [(True, 1.0), (False, 1.8), (True, 1.8)])
def test_logits_are_processed_before_they_are_normalised(cuda_ok, masked, rep):
    import paged_decode as ex
    g = torch.Generator(device="cuda").manual_seed(3)
    lens, steps = [7, 150, 64, 20, 97, 33], 4
    model = ex.Model(L=2, Hq=8, Hkv=2, D=64, V=V, rows=max(lens) + steps, seed=2)
    r = torch.rand((B, N), device="cuda", generator=g).clamp(min=0.05)
    pen = torch.tensor([[rep, 0.3, 0.2]] * B, device="cuda")
    mask = None
    if masked:  # a third of the tokens
        bits = np.random.default_rng(4).random((B, (V + 31) // 32 * 32)) < 1 / 3
        mask = torch.from_numpy(np.packbits(bits, axis=1, bitorder="little").view("<i4").copy()).cuda()
    loop = ex.Loop(model, B, N, lens, steps, torch.full((B, N), BETA, device="cuda"), r, gamma=GAMMA, penalties=pen,
                   mask=mask)
    loop.load_documents(torch.randn((sum(lens), model.Hq * model.D), device="cuda", generator=g))
    loop.history[:, :3] = torch.arange(3, dtype=torch.int32, device="cuda") * 7
    loop.n_history += 3
    loop.t = 3
    w = model.unembed.double().cpu().numpy()
    history, n_history = loop.history.cpu().numpy(), loop.n_history.cpu().numpy()
    token, expert = loop.step()
    h = ref.f64(loop.hidden)
    z, mag = ref.process(h @ w.T, N + 1, history=history, history_len=n_history, penalties=pen.cpu().numpy(),
                         mask=None if mask is None else mask.cpu().numpy())
    top = z.max(axis=1, keepdims=True)
    want = z - top - np.log(np.exp(z - top).sum(axis=1, keepdims=True))
    # a logit is a sum of d products in fp32 (d 2^-24 of their magnitudes); it and its row's log-sum-exp are rounded a
    # few times on the way, the penalty may scale it by `rep`, and the second sum takes as much again
    e = (h.shape[1] * 2.0 ** -24 * (np.abs(h) @ np.abs(w).T).max() + 8 * 2.0 ** -24 * mag.max()) * max(rep, 1) * 2
    got = loop.logprobs.double().cpu().numpy()
    assert np.array_equal(np.isneginf(got), np.isneginf(want))
    fin = np.isfinite(want)
    assert np.abs(got - want)[fin].max() <= e
    tok, exp, lead = choice(want, r.double().cpu().numpy())
    for b in range(B):
        if lead[b] > 8 * e:
            assert (int(token[b]), int(expert[b])) == (tok[b], exp[b])
