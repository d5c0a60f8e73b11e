"""A PagedCache holds the tensors whose addresses it has taken (no GPU needed)."""
import pytest
import torch


@pytest.fixture(scope="module")
def make():
    from paper_2601_08670_gb300 import build
    build.build()
    import paper_2601_08670_gb300 as pced

    def cache(**kw):
        k = torch.zeros((4, 2, 16, 64), dtype=torch.bfloat16)
        return pced.PagedCache(k, k.clone(), torch.zeros((3, 2), dtype=torch.int32), torch.ones(3, dtype=torch.int32),
                               **kw)
    return cache


@pytest.mark.parametrize("name", ["k", "v", "block_table", "seq_len", "summary", "key_step"])
def test_other_tensors_are_refused(make, name):
    # the calls would go on with the old addresses, whose memory may have gone back to the allocator
    cache = make(summary=torch.zeros((4, 2, 2, 64), dtype=torch.int8), key_step=torch.ones(2))
    held = getattr(cache, name)
    with pytest.raises(AttributeError, match=name):
        setattr(cache, name, held.clone())
    assert getattr(cache, name) is held and getattr(cache.struct, name) == held.data_ptr()


def test_a_summary_given_later_is_refused(make):
    cache = make()
    with pytest.raises(AttributeError, match="summary"):
        cache.summary = torch.zeros((4, 2, 2, 64), dtype=torch.int8)
    with pytest.raises(AttributeError, match="k"):
        del cache.k


@pytest.mark.parametrize("name", ["num_blocks", "block_rows", "max_blocks", "S", "Hkv", "D"])
def test_sizes_are_refused(make, name):
    with pytest.raises(AttributeError, match=name):
        setattr(make(), name, 1 << 20)


def test_contents_change_in_place(make):
    cache = make()
    cache.seq_len += 1  # the tensor itself, put back where it was
    cache.k[2] = 1.0
    assert cache.seq_len.tolist() == [2, 2, 2] and cache.struct.seq_len == cache.seq_len.data_ptr()
