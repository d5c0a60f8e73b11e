"""Which fields of a PagedCache and of a PagedCache8 take no other tensor (host side; nothing is launched)."""
import pytest
import torch


def make(pced, eight):
    k = torch.zeros(3, 2, 16, 64, dtype=torch.float8_e4m3fn if eight else torch.bfloat16)
    more = [torch.ones(3, 2, 2)] if eight else []
    return (pced.PagedCache8 if eight else pced.PagedCache)(k, k.clone(), *more, torch.zeros(2, 4, dtype=torch.int32),
                                                            torch.zeros(2, dtype=torch.int32))


def test_a_bf16_cache_has_no_scale_of_its_own():
    # what a program keeps there is the program's
    import paper_2601_08670_gb300 as pced
    c = make(pced, False)
    c.scale = 0.5
    c.scale = 0.25
    assert c.scale == 0.25
    del c.scale
    assert not hasattr(c, "scale")


def test_an_8_bit_caches_scale_stays():
    import paper_2601_08670_gb300 as pced
    c = make(pced, True)
    with pytest.raises(AttributeError, match="scale"):
        c.scale = torch.ones(3, 2, 2)
    with pytest.raises(AttributeError, match="scale"):
        del c.scale
    c.scale *= 2  # in place: the same tensor put back
    assert c.struct8.scale == c.scale.data_ptr() and float(c.scale[0, 0, 0]) == 2
    for name in ("k", "seq_len"):
        with pytest.raises(AttributeError, match=name):
            setattr(c, name, getattr(c, name).clone())
