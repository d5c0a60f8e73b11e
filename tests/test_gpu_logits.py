"""logits_process against its definition in 64 bits: a few roundings to fp32, masked entries exactly -inf."""
import numpy as np
import pytest
import torch

import paged_ref as ref

pytestmark = pytest.mark.gpu


def run(B, R, V, n_hist=0, n_bias=0, masks=0, mask_row=True, pad=0, in_place=False, shift=0, seed=0, edit=None, status=0):
    import paper_2601_08670_gb300 as pced
    rng = np.random.default_rng([seed, B, R, V])
    x = rng.normal(0, 3, size=(B * R, V)).astype(np.float32)
    a = {}
    if n_hist:
        a["history"] = rng.integers(0, min(V, 3 * n_hist), size=(B, n_hist)).astype(np.int32)
        a["history_len"] = rng.integers(0, n_hist + 1, size=B).astype(np.int32)
        a["history_len"][0] = n_hist
        a["penalties"] = np.stack([rng.uniform(0.8, 1.6, B), rng.uniform(-0.5, 1, B), rng.uniform(-0.5, 1, B)],
                                  axis=1).astype(np.float32)
    if n_bias:
        a["bias_ids"] = rng.integers(-1, V, size=(B, n_bias)).astype(np.int32)
        a["bias"] = rng.normal(0, 4, size=(B, n_bias)).astype(np.float32)
    if masks:
        a["mask"] = rng.integers(-2 ** 31, 2 ** 31, size=(masks, (V + 31) // 32 + 1)).astype(np.int32)
        if mask_row:
            a["mask_row"] = rng.integers(-1, masks, size=B).astype(np.int32)
    if edit:
        edit(x, a)
    want, mag = ref.process(x, R, **{k: (np.clip(v, 0, n_hist) if k == "history_len" else v) for k, v in a.items()})
    # rows `pad` entries further apart than V, the first `shift` entries from an aligned address
    buf = torch.full((B * R * (V + pad) + shift,), 7.0, device="cuda")
    view = torch.as_strided(buf, (B * R, V), (V + pad, 1), shift)
    view.copy_(torch.from_numpy(x))
    args = {k: torch.from_numpy(v).cuda() for k, v in a.items()}
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = pced.logits_process(view, R, out=view if in_place else None, status=st, **args)
    torch.cuda.synchronize()
    assert int(st.item()) == status
    if not in_place:
        assert np.array_equal(view.cpu().numpy(), x, equal_nan=True)
    if pad:
        gaps = torch.as_strided(buf, (B * R - 1, pad), (V + pad, 1), shift + V)
        assert bool((gaps == 7.0).all())
    got = got.cpu().numpy().astype(np.float64)
    assert np.array_equal(np.isneginf(got), np.isneginf(want))
    assert np.array_equal(np.isnan(got), np.isnan(want))
    fin = np.isfinite(want)
    assert np.array_equal(got[~fin & ~np.isnan(want)], want[~fin & ~np.isnan(want)])
    # five roundings to fp32 at most, each of a value no larger than mag
    assert np.all(np.abs(got - want)[fin] <= 5 * 2.0 ** -24 * mag[fin])


@pytest.mark.parametrize("V", [1, 31, 1000, 2047, 2048, 2049, 5004, 20_011])
@pytest.mark.parametrize("B,R", [(1, 1), (1, 9), (3, 4)])
def test_everything_at_once(cuda_ok, V, B, R):
    run(B, R, V, n_hist=200, n_bias=20, masks=4)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("pad,shift", [(0, 0), (0, 1), (4, 0), (3, 0), (60, 2)])
def test_strides_and_alignment(cuda_ok, pad, shift, in_place):
    run(2, 3, 4100, n_hist=50, n_bias=5, masks=2, pad=pad, shift=shift, in_place=in_place)


def test_each_alone_and_none(cuda_ok):
    run(2, 3, 3000)
    run(2, 3, 3000, n_hist=1)
    run(2, 3, 3000, n_bias=1)
    run(2, 3, 3000, masks=2, mask_row=False)
    run(16, 17, 3000, masks=1)


def test_a_vocabulary_and_a_long_history(cuda_ok):
    run(2, 9, 128256, n_hist=8192, n_bias=300, masks=3)


def test_many_rows(cuda_ok):
    run(1, 272, 5000, n_hist=64)
    run(100, 2, 2500, n_hist=64, masks=5)


def test_infinities_and_nan_pass_through(cuda_ok):
    def edit(x, a):
        x[:, :6] = [np.inf, -np.inf, np.nan, 0.0, -0.0, 3.4e38]
        a["history"][:, :8] = [0, 1, 2, 3, 4, 5, 5, 5]
        a["penalties"][:, 0] = 1.25
        a["bias_ids"][:, 0], a["bias"][:, 0] = 9, -np.inf
    run(2, 2, 1000, n_hist=30, n_bias=4, edit=edit)


def test_mask_that_forbids_everything(cuda_ok):
    run(2, 2, 1000, masks=2, edit=lambda x, a: a["mask"].fill(0))


def test_last_bias_of_a_token_counts(cuda_ok):
    def edit(x, a):
        a["bias_ids"][:] = [5, 7, 5, -1, 7, 5]
    run(3, 2, 100, n_bias=6, edit=edit)


def test_bad_numbers_are_left_out_and_flagged(cuda_ok):
    import paper_2601_08670_gb300 as pced

    def tok(x, a):
        a["history"][0, :2] = [-2, 1000]
    run(2, 2, 1000, n_hist=9, edit=tok, status=pced.PCED_DEV_BAD_TOKEN)
    run(2, 2, 1000, n_hist=9, edit=lambda x, a: a["history"].__setitem__((0, 3), -1))
    run(2, 2, 1000, n_bias=9, edit=lambda x, a: a["bias_ids"].__setitem__((1, 3), 1000), status=pced.PCED_DEV_BAD_TOKEN)
    run(2, 2, 1000, n_hist=9, edit=lambda x, a: a["history_len"].__setitem__(slice(None), [10, -1]),
        status=pced.PCED_DEV_BAD_LENGTH)
    run(2, 2, 1000, masks=3, edit=lambda x, a: a["mask_row"].__setitem__(slice(None), [3, -2]),
        status=pced.PCED_DEV_BAD_INDEX)


def test_masked_tokens_are_never_chosen(cuda_ok):
    # the whole of a choice: masked rows of experts and amateur through Eq. 2 and Eq. 3
    import paper_2601_08670_gb300 as pced
    g = torch.Generator(device="cuda").manual_seed(1)
    B, N, V = 2, 3, 5000
    lp = torch.log_softmax(torch.randn((B * (N + 1), V), device="cuda", generator=g) * 4, dim=1)
    allowed = [17, 4000]
    mask = torch.zeros((2, (V + 31) // 32), dtype=torch.int32, device="cuda")
    for b, v in enumerate(allowed):
        mask[b, v // 32] = 1 << (v % 32)
    beta, r = torch.full((B, N), 0.5, device="cuda"), torch.full((B, N), 0.7, device="cuda")
    y = pced.logits_process(lp, N + 1, mask=mask)
    token, expert, _ = pced.contrastive_select(y, beta, r, 2.5)
    s = 1.5 * lp.view(B, N + 1, V)[:, 1:] - 0.5 * lp.view(B, N + 1, V)[:, :1]
    for b, v in enumerate(allowed):
        assert int(token[b]) == v and int(expert[b]) == int(s[b, :, v].argmax()) + 1
