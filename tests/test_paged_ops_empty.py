"""Tensors without elements are refused, not taken for arguments that were not given (no GPU needed: the checks come
before anything is launched)."""
import pytest
import torch

bf, i32 = torch.bfloat16, torch.int32


@pytest.fixture(scope="module")
def pced():
    from paper_2601_08670_gb300 import build
    build.build()
    import paper_2601_08670_gb300 as pced
    return pced


@pytest.fixture(scope="module")
def cache(pced):
    k = torch.zeros((4, 2, 16, 64), dtype=bf)
    return pced.PagedCache(k, k.clone(), torch.zeros((3, 2), dtype=i32), torch.ones(3, dtype=i32))


@pytest.mark.parametrize("sel", [torch.zeros((3, 2, 0), dtype=i32), torch.zeros((3, 2, 4), dtype=i32)[:, :, :0]])
def test_a_selection_without_places_is_not_all_blocks(pced, cache, sel):
    q = torch.zeros((3, 8, 64), dtype=bf)
    with pytest.raises(ValueError, match="sel"):
        pced.paged_attention(cache, q, sel=sel, ws=torch.zeros(1 << 22, dtype=torch.uint8))


@pytest.mark.parametrize("T", [0, 3])
def test_a_rotation_table_without_rows_is_not_no_rotation(pced, cache, T):
    kv = torch.zeros((T, 2, 64), dtype=bf)
    with pytest.raises(ValueError, match="rope"):
        pced.kv_append(cache, None, kv, kv, rope=torch.zeros((0, 64)), tok_start=torch.zeros(4, dtype=i32))


@pytest.mark.parametrize("shape", [(0, 1), (2, 0), (0, 0)])
@pytest.mark.parametrize("mask_row", [None, torch.zeros(2, dtype=i32)])
def test_masks_without_rows_or_words_are_not_no_mask(pced, shape, mask_row):
    with pytest.raises(ValueError, match="mask"):
        pced.logits_process(torch.zeros(4, 8), 2, mask=torch.zeros(shape, dtype=i32), mask_row=mask_row)


def test_empty_histories_and_biases_stay_none(pced):
    # nothing to count and nothing to add: right in everything but where the tensors lie
    with pytest.raises(ValueError, match="CUDA"):
        pced.logits_process(torch.zeros(4, 8), 2, history=torch.zeros((2, 0), dtype=i32),
                            history_len=torch.zeros(2, dtype=i32), penalties=torch.ones(2, 3),
                            bias_ids=torch.zeros((2, 0), dtype=i32), bias=torch.zeros(2, 0))


def test_a_status_word_has_one(pced, cache):
    kv = torch.zeros((3, 2, 64), dtype=bf)
    with pytest.raises(ValueError, match="status"):
        pced.kv_append(cache, None, kv, kv, status=torch.zeros(0, dtype=i32))
