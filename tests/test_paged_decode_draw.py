"""Tokens in the example's loop: a query whose mask forbids everything has no token, and the others theirs."""
import os
import sys

import numpy as np
import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))


def test_draw_without_a_token(monkeypatch):
    # -1, as the operator answers for a row without a token, names no score (on the host: no GPU needed)
    import paged_decode as ex
    B, N, V = 2, 2, 5
    loop = ex.Loop.__new__(ex.Loop)
    loop.B, loop.N, loop.gamma, loop.status, loop.sampling = B, N, 2.5, None, {}
    loop.beta, loop.r, loop.random = torch.full((B, N), 0.5), torch.tensor([[0.9, 0.2]] * B), torch.Generator()
    lp = torch.zeros((B * (N + 1), V)).log_softmax(1)
    lp[:N + 1] = float("nan")  # a softmax of nothing but -inf
    monkeypatch.setattr(ex.pced, "sample", lambda *a, **kw: torch.tensor([-1, 3], dtype=torch.int32))
    token, expert = loop.draw(lp)
    assert token.tolist() == [-1, 3] and expert.tolist() == [0, 1] and expert.dtype == torch.int32


@pytest.mark.gpu
@pytest.mark.parametrize("eight,sampling", [(False, dict(temperature=0.8, top_p=0.9)), (True, dict(temperature=0.8)),
                                            (False, None)])
def test_a_query_whose_mask_forbids_everything(cuda_ok, eight, sampling):
    import paged_decode as ex
    B, N, V, steps = 2, 2, 1000, 3
    lens = [7, 150, 64, 20, 97, 33]
    model = ex.Model(L=2, Hq=8, Hkv=2, D=64, V=V, rows=max(lens) + steps)
    r = torch.tensor([[0.9, 0.2], [0.4, 0.7]], device="cuda")
    hidden = torch.randn((sum(lens), model.Hq * model.D), device="cuda", generator=torch.Generator("cuda").manual_seed(3))
    allowed = np.full((B, (V + 31) // 32), -1, np.int32)
    allowed[0] = 0
    loops = []
    for mask in (torch.from_numpy(allowed).cuda(), torch.full((B, (V + 31) // 32), -1, dtype=torch.int32, device="cuda")):
        loop = ex.Loop(model, B, N, lens, steps, torch.full((B, N), 0.5, device="cuda"), r, mask=mask, eight=eight,
                       sampling=sampling)
        loop.load_documents(hidden)
        for _ in range(steps):
            loop.step()
        assert loop.device_status() == 0
        loops.append(loop)
    barred, free = loops
    assert barred.history[0].tolist() == [-1] * steps and barred.expert[0].tolist() == [0] * steps
    # the other query decodes as it does beside one with tokens
    assert torch.equal(barred.history[1], free.history[1]) and torch.equal(barred.expert[1], free.expert[1])
    assert bool((free.history >= 0).all()) and bool((free.expert >= 1).all())
