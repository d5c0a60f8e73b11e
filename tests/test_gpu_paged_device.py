"""The calls over paged caches run on the device of their tensors or not at all."""
import types

import pytest
import torch

pytestmark = pytest.mark.gpu


def make():
    import paper_2601_08670_gb300 as pced
    k = torch.ones((4, 2, 16, 64), dtype=torch.bfloat16, device="cuda")
    return pced.PagedCache(k, k.clone(), torch.zeros((1, 2), dtype=torch.int32, device="cuda"),
                           torch.full((1,), 16, dtype=torch.int32, device="cuda"),
                           summary=torch.zeros((4, 2, 2, 64), dtype=torch.int8, device="cuda"),
                           key_step=torch.ones(2, device="cuda"))


def test_a_device_that_is_not_the_current_one(cuda_ok):
    import paper_2601_08670_gb300 as pced
    cache = make()
    cache.gpu += 1  # as if its tensors lay on the next device (the call has no other tensor that tells)
    with pytest.raises(ValueError, match="current"):
        pced.block_summaries(cache)
    torch.cuda.synchronize()
    assert not cache.summary.any()


def test_a_stream_of_another_device(cuda_ok):
    import paper_2601_08670_gb300 as pced
    cache = make()
    other = types.SimpleNamespace(cuda_stream=torch.cuda.current_stream().cuda_stream, device_index=1)
    with pytest.raises(ValueError, match="stream"):
        pced.block_summaries(cache, stream=other)
    with pytest.raises(ValueError, match="stream"):
        pced.logits_process(torch.zeros((2, 8), device="cuda"), 2, out=torch.zeros((2, 8), device="cuda"), stream=other)
    torch.cuda.synchronize()
    assert not cache.summary.any()


def test_a_stream_that_has_no_handle(cuda_ok):
    # an error, and nothing launched on the default stream in its place
    import paper_2601_08670_gb300 as pced
    cache = make()
    with pytest.raises(TypeError):
        pced.block_summaries(cache, stream=types.SimpleNamespace(cuda_stream="7", device_index=0))
    torch.cuda.synchronize()
    assert not cache.summary.any()


def test_streams_of_this_device(cuda_ok):
    import paper_2601_08670_gb300 as pced
    cache = make()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for s in (side, torch.cuda.current_stream(), torch.cuda.default_stream(),
              torch.cuda.ExternalStream(side.cuda_stream)):
        cache.summary.zero_()
        torch.cuda.synchronize()
        pced.block_summaries(cache, stream=s)
        torch.cuda.synchronize()
        assert int(cache.summary[0].max()) == 1
