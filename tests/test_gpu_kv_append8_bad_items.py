"""kv_append into 8-bit caches where a sequence's length, table or starts are bad: the other sequence's row is appended, as if
it were alone, and nothing else changes, to the last byte of keys, values, scales and summaries."""
import numpy as np
import pytest
import torch

import cache8_ref as ref8
import paged_ref as ref

pytestmark = pytest.mark.gpu
LENGTH, BLOCK = "PCED_DEV_BAD_LENGTH", "PCED_DEV_BAD_BLOCK"


# (lengths, table entries, starts, condition, whether the second sequence gets its row)
@pytest.mark.parametrize("lens,table,start,bit,second", [
    ([200, 3], {}, None, LENGTH, True), ([-1, 3], {}, None, LENGTH, True), ([40, 3], {(0, 0): 99}, None, BLOCK, True),
    ([40, 3], {(0, 0): 99}, [0, 1, 2], BLOCK, True), ([40, 3], {(0, 0): -7}, [0, 1, 2], BLOCK, True),
    ([200, 3], {}, [0, 1, 2], LENGTH, True), ([-1, 3], {}, [0, 1, 2], LENGTH, True), ([0, 3], {}, [0, 1, 2], LENGTH, True),
    # from where the starts fall on, tokens could be named twice
    ([40, 3], {}, [0, -1, 2], LENGTH, False), ([40, 3], {}, [0, 5, 2], LENGTH, False)])
@pytest.mark.parametrize("heads", [(8, 2, 64), (32, 8, 128)])
def test_the_other_sequence_alone(cuda_ok, heads, lens, table, start, bit, second):
    import paper_2601_08670_gb300 as pced
    Hq, Hkv, D = heads
    rng = np.random.default_rng(2)
    c = ref8.make_cache(rng, [40, 3], Hkv, D, 64, spoil=False)
    c["table"] = c["table"][:, :1].copy()
    for at, b in table.items():
        c["table"][at] = b
    c["lens"] = np.array(lens, np.int32)
    summary = rng.integers(-60, 61, size=(len(c["k"]), Hkv, 2, D)).astype(np.int8)
    cache = ref8.to_device(c, summary)
    x = ref.rng_bf16(rng, (2, Hq + 2 * Hkv, D), 30.0)  # (larger than the scales: the second's two rows move)
    dev, status = x.cuda(), torch.zeros(1, dtype=torch.int32, device="cuda")
    q_out = pced.kv_append(cache, dev[:, :Hq], dev[:, Hq:Hq + Hkv], dev[:, Hq + Hkv:], status=status,
                           tok_start=None if start is None else torch.tensor(start, dtype=torch.int32, device="cuda"))
    assert int(status.item()) == getattr(pced, bit)
    h = x.float().numpy()[1:]
    want, want_summary = ref8.append(c, h[:, Hq:Hq + Hkv], h[:, Hq + Hkv:], [0, 1 if second else 0], summary)
    assert np.array_equal(cache.scale.cpu().numpy(), want["scale"])
    assert np.array_equal(cache.summary.cpu().numpy(), want_summary)
    for name in ("k", "v"):
        assert np.array_equal(getattr(cache, name).view(torch.uint8).cpu().numpy(), want[name]), name
    if second:
        b = c["table"][1, 0]
        assert (want["scale"][b] != c["scale"][b]).any() and (want["k"][b, :, 2] != c["k"][b, :, 2]).any()
        assert torch.equal(q_out[1], dev[1, :Hq])
