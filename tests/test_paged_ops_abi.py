"""What the operators over paged caches refuse before they touch a device (no GPU needed: every call here fails
host-side validation), and the checks of the binding."""
import ctypes

import pytest
import torch

FAKE = 1 << 12  # non-null, aligned; never dereferenced because validation fails first
INVALID, WORKSPACE, UNSUPPORTED = 1, 2, 3


@pytest.fixture(scope="module")
def pced():
    from paper_2601_08670_gb300 import build
    build.build()
    import paper_2601_08670_gb300 as pced
    return pced


def cache(pced, **kw):
    c = pced.PagedCacheStruct(FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 100, 64, 10, 3, 2, 64)
    for k, v in kw.items():
        setattr(c, k, v)
    return ctypes.byref(c)


BAD_CACHES = [(dict(block_table=None), INVALID), (dict(seq_len=None), INVALID), (dict(S=0), INVALID),
              (dict(Hkv=0), INVALID), (dict(num_blocks=0), INVALID), (dict(max_blocks=0), INVALID),
              (dict(block_rows=24), INVALID), (dict(block_rows=0), INVALID), (dict(k=FAKE + 2), INVALID),
              (dict(summary=FAKE + 8), INVALID), (dict(D=96), UNSUPPORTED), (dict(S=1025), UNSUPPORTED),
              (dict(num_blocks=1 << 30), UNSUPPORTED)]


def calls(pced, c):
    """Every call over a cache, its other arguments valid."""
    L = pced.lib()
    return [L.pced_kv_append(c, FAKE, 512, FAKE, 128, FAKE, 128, FAKE, 8, None, 3, FAKE, 10, None, FAKE, None),
            L.pced_block_summaries(c, FAKE, None),
            L.pced_block_select(c, FAKE, 512, 8, 4, 1, 1, FAKE, FAKE, None),
            L.pced_paged_attention(c, FAKE, 512, 8, None, 0, 0, 0.1, FAKE, 0, FAKE, FAKE, 1 << 30, None)]


@pytest.mark.parametrize("kw,code", BAD_CACHES)
def test_bad_caches(pced, kw, code):
    assert calls(pced, cache(pced, **kw)) == [code] * 4


def test_null_cache(pced):
    assert calls(pced, None) == [INVALID] * 4


@pytest.mark.skipif(torch.cuda.is_available(), reason="only meaningful without a GPU")
def test_valid_calls_without_a_device(pced):
    assert calls(pced, cache(pced)) == [5] * 4
    assert pced.lib().pced_logits_process(FAKE, FAKE, 100, 1, 2, 100, None, 0, None, None, None, None, 0, None, 0, 0,
                                          None, None, None) == 5


def test_append_refusals(pced):
    f = pced.lib().pced_kv_append
    good = [cache(pced), FAKE, 512, FAKE, 128, FAKE, 128, FAKE, 8, None, 3, FAKE, 10, None, FAKE, None]

    def with_(**kw):
        a = list(good)
        for i, v in kw.items():
            a[int(i[1:])] = v
        return f(*a)
    assert with_(_1=None) == INVALID              # queries in but not out
    assert with_(_1=None, _7=None) == INVALID     # Hq without queries
    assert with_(_3=None) == INVALID and with_(_5=None) == INVALID
    assert with_(_2=511) == INVALID and with_(_2=504) == INVALID and with_(_4=120) == INVALID
    assert with_(_6=132) == INVALID and with_(_3=FAKE + 2) == INVALID and with_(_7=FAKE + 8) == INVALID
    assert with_(_8=9) == INVALID and with_(_8=0) == INVALID
    assert with_(_8=18, _2=2000) == UNSUPPORTED   # nine query heads per kv-head
    assert with_(_10=4) == INVALID                # T is not S
    assert with_(_9=FAKE, _10=-1) == INVALID
    assert with_(_12=0) == INVALID                # empty rotation table
    assert with_(_9=FAKE, _10=0) == 0             # nothing to append
    assert with_(_0=cache(pced, key_step=None)) == INVALID
    assert with_(_0=cache(pced, v=None)) == INVALID


def test_summaries_and_select_refusals(pced):
    L = pced.lib()
    for kw in (dict(k=None), dict(summary=None), dict(key_step=None)):
        assert L.pced_block_summaries(cache(pced, **kw), None, None) == INVALID
    f = L.pced_block_select
    assert f(cache(pced, summary=None), FAKE, 512, 8, 4, 1, 1, FAKE, None, None) == INVALID
    assert f(cache(pced), None, 512, 8, 4, 1, 1, FAKE, None, None) == INVALID
    assert f(cache(pced), FAKE, 512, 8, 4, 1, 1, None, None, None) == INVALID
    assert f(cache(pced), FAKE, 510, 8, 4, 1, 1, FAKE, None, None) == INVALID
    assert f(cache(pced), FAKE, 512, 8, 4, 3, 2, FAKE, None, None) == INVALID   # more forced than wanted
    assert f(cache(pced), FAKE, 512, 8, 0, 0, 0, FAKE, None, None) == INVALID
    assert f(cache(pced), FAKE, 512, 8, 4, -1, 1, FAKE, None, None) == INVALID
    assert f(cache(pced, max_blocks=1 << 20), FAKE, 512, 8, 4, 1, 1, FAKE, None, None) == UNSUPPORTED


def test_attention_refusals(pced):
    L = pced.lib()
    f = lambda c=None, q=FAKE, stride=512, Hq=8, sel=None, n=0, rows=0, scale=0.1, out=FAKE, kind=0, ws=FAKE, \
        size=1 << 30: L.pced_paged_attention(c or cache(pced), q, stride, Hq, sel, n, rows, scale, out, kind, None, ws,
                                             size, None)
    assert f(c=cache(pced, k=None)) == INVALID and f(q=None) == INVALID and f(out=None) == INVALID
    assert f(ws=None) == INVALID and f(out=FAKE + 4) == INVALID
    assert f(stride=100) == INVALID and f(Hq=7) == INVALID and f(Hq=18, stride=4096) == UNSUPPORTED
    assert f(sel=FAKE, n=0) == INVALID and f(n=3) == INVALID
    assert f(rows=-1) == INVALID and f(scale=float("nan")) == INVALID and f(kind=2) == INVALID
    assert f(size=16) == WORKSPACE and f(ws=FAKE + 16) == WORKSPACE
    assert b"workspace" in L.pced_last_error()
    assert L.pced_paged_attention_workspace_size(3, 7, 2, 64) == 0
    assert L.pced_paged_attention_workspace_size(3, 8, 2, 64) >= 256


def test_logits_refusals(pced):
    f = pced.lib().pced_logits_process
    good = dict(x=FAKE, y=FAKE, stride=100, B=2, R=3, V=100, hist=FAKE, hs=10, hl=FAKE, pen=FAKE, ids=FAKE, bias=FAKE,
                nb=3, mask=FAKE, nm=2, words=4, row=FAKE, status=FAKE, stream=None)
    bad = [dict(x=None), dict(y=None), dict(stride=99), dict(B=0), dict(R=0), dict(V=0), dict(B=70_000), dict(hs=0),
           dict(hl=None), dict(pen=None), dict(hist=None), dict(ids=None), dict(bias=None), dict(nb=0), dict(nb=-1),
           dict(nm=0), dict(words=3), dict(row=None, nm=1), dict(mask=None), dict(x=FAKE + 2), dict(status=FAKE + 1)]
    for kw in bad:
        assert f(*dict(good, **kw).values()) == INVALID, kw


def test_binding_refuses_bad_tensors(pced):
    bf, i32 = torch.bfloat16, torch.int32
    k = torch.zeros((4, 2, 16, 64), dtype=bf)
    table, lens = torch.zeros((3, 2), dtype=i32), torch.zeros(3, dtype=i32)
    summ, step = torch.zeros((4, 2, 2, 64), dtype=torch.int8), torch.ones(2)
    ok = pced.PagedCache(k, k.clone(), table, lens, summary=summ, key_step=step)
    for args, kw in [((k.float(), k, table, lens), {}), ((k, k[:3], table, lens), {}), ((k, k, table.long(), lens), {}),
                     ((k, k, table, lens[:2]), {}), ((None, None, table, lens), {}),
                     ((k, k, table, lens), dict(block_rows=32)), ((k, k, table, lens), dict(summary=summ[:, :1])),
                     ((k, k, table, lens), dict(key_step=step[:1])), ((k.transpose(0, 1), k, table, lens), {})]:
        with pytest.raises(ValueError):
            pced.PagedCache(*args, **kw)
    q, kv = torch.zeros((3, 8, 64), dtype=bf), torch.zeros((3, 2, 64), dtype=bf)
    bad = [lambda: pced.kv_append(ok, q.float(), kv, kv), lambda: pced.kv_append(ok, q, kv[:, :1], kv),
           lambda: pced.kv_append(ok, q[:2], kv, kv), lambda: pced.kv_append(ok, q, kv, kv[:2]),
           lambda: pced.kv_append(ok, q, kv, kv, rope=torch.zeros((4, 32))),
           lambda: pced.kv_append(ok, q, kv, kv, tok_start=table[0]),
           lambda: pced.kv_append(ok, q, kv, kv, positions=lens.long()),
           lambda: pced.kv_append(ok, None, kv, kv, q_out=q),
           lambda: pced.kv_append(ok, q.transpose(0, 1).contiguous().transpose(0, 1), kv, kv),
           lambda: pced.block_select(ok, q[:2], 4), lambda: pced.block_select(ok, q, 4, sel=torch.zeros((3, 2, 5), dtype=i32)),
           lambda: pced.paged_attention(ok, q[:2]), lambda: pced.paged_attention(ok, q, sel=table),
           lambda: pced.paged_attention(ok, q, out=q.double()), lambda: pced.paged_attention(ok, q, lse=torch.zeros(3, 7)),
           lambda: pced.logits_process(torch.zeros(4, 8).double(), 2), lambda: pced.logits_process(torch.zeros(4, 8), 3),
           lambda: pced.logits_process(torch.zeros(4, 8).t(), 2),
           lambda: pced.logits_process(torch.zeros(4, 8), 2, history=torch.zeros((2, 3), dtype=i32)),
           lambda: pced.logits_process(torch.zeros(4, 8), 2, penalties=torch.zeros((2, 3))),
           lambda: pced.logits_process(torch.zeros(4, 8), 2, bias=torch.zeros((2, 3))),
           lambda: pced.logits_process(torch.zeros(4, 8), 2, mask_row=lens[:2]),
           lambda: pced.logits_process(torch.zeros(4, 8), 2, mask=torch.zeros((2, 1))),
           lambda: pced.logits_process(torch.zeros(4, 8), 2, out=torch.zeros(4, 9)[:, :8])]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {i} was accepted")


def test_binding_refuses_tensors_off_the_gpu(pced):
    # right in everything but where they lie: host memory is never handed to a kernel
    bf, i32 = torch.bfloat16, torch.int32
    k = torch.zeros((4, 2, 16, 64), dtype=bf)
    c = pced.PagedCache(k, k.clone(), torch.zeros((3, 2), dtype=i32), torch.ones(3, dtype=i32),
                        summary=torch.zeros((4, 2, 2, 64), dtype=torch.int8), key_step=torch.ones(2))
    q, kv = torch.zeros((3, 8, 64), dtype=bf), torch.zeros((3, 2, 64), dtype=bf)
    ws = torch.zeros(1 << 22, dtype=torch.uint8)
    for call in (lambda: pced.kv_append(c, q, kv, kv), lambda: pced.block_summaries(c),
                 lambda: pced.block_select(c, q, 4), lambda: pced.paged_attention(c, q, ws=ws),
                 lambda: pced.logits_process(torch.zeros(4, 8), 2)):
        with pytest.raises(ValueError, match="CUDA"):
            call()


def test_binding_refuses_what_is_no_tensor_or_number(pced):
    k = torch.zeros((4, 2, 16, 64), dtype=torch.bfloat16)
    c = pced.PagedCache(k, k, torch.zeros((3, 2), dtype=torch.int32), torch.ones(3, dtype=torch.int32))
    q = torch.zeros((3, 8, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        pced.kv_append(c, None, [1, 2], q[:, :2])
    with pytest.raises(ValueError):
        pced.block_select(c, q, 1 << 40, sel=torch.zeros((3, 2, 4), dtype=torch.int32))
    with pytest.raises(TypeError):
        pced.block_select(c, q, 4.5, sel=torch.zeros((3, 2, 4), dtype=torch.int32))
    with pytest.raises(ValueError):
        pced.paged_attention(c, q, total_rows=1, out=q.half(), ws=torch.zeros(256, dtype=torch.uint8))
