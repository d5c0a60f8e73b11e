"""What the operators over 8-bit caches and sample refuse before they touch a device (no GPU needed), and what a
PagedCache8 holds."""
import ctypes
import glob
import os
import re

import pytest
import torch

FAKE = 1 << 12  # non-null, aligned; never dereferenced because validation fails first
INVALID, WORKSPACE, UNSUPPORTED, NO_DEVICE = 1, 2, 3, 5
bf, f8, i32 = torch.bfloat16, torch.float8_e4m3fn, torch.int32
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def pced():
    from paper_2601_08670_gb300 import build
    build.build()
    import paper_2601_08670_gb300 as pced
    return pced


def cache(pced, scale=FAKE, **kw):
    c = pced.PagedCacheStruct(FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 100, 64, 10, 3, 2, 64)
    for k, v in kw.items():
        setattr(c, k, v)
    return ctypes.byref(pced.PagedCache8Struct(c, scale))


def calls(pced, c):
    L = pced.lib()
    return [L.pced_kv_append8(c, FAKE, 512, FAKE, 128, FAKE, 128, FAKE, 8, None, 3, FAKE, 10, None, FAKE, None),
            L.pced_paged_attention8(c, FAKE, 512, 8, None, 0, 0, 0.1, FAKE, 0, FAKE, FAKE, 1 << 30, None)]


@pytest.mark.parametrize("kw,code", [
    (dict(scale=None), INVALID), (dict(scale=FAKE + 4), INVALID), (dict(block_table=None), INVALID),
    (dict(seq_len=None), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(S=0), INVALID),
    (dict(block_rows=24), INVALID), (dict(k=FAKE + 8), INVALID), (dict(D=96), UNSUPPORTED), (dict(S=1025), UNSUPPORTED),
    (dict(num_blocks=1 << 30), UNSUPPORTED)])
def test_bad_caches(pced, kw, code):
    assert calls(pced, cache(pced, **kw)) == [code] * 2


def test_null_cache(pced):
    assert calls(pced, None) == [INVALID] * 2


@pytest.mark.skipif(torch.cuda.is_available(), reason="only meaningful without a GPU")
def test_valid_calls_without_a_device(pced):
    assert calls(pced, cache(pced)) == [NO_DEVICE] * 2
    assert pced.lib().pced_sample(FAKE, 0, 100, 2, 100, FAKE, None, None, None, None, FAKE, None, None, None) == NO_DEVICE


def test_append_and_attention_arguments(pced):
    f = pced.lib().pced_kv_append8
    good = [cache(pced), FAKE, 512, FAKE, 128, FAKE, 128, FAKE, 8, None, 3, FAKE, 10, None, FAKE, None]

    def with_(**kw):
        a = list(good)
        for i, v in kw.items():
            a[int(i[1:])] = v
        return f(*a)
    assert with_(_1=None) == INVALID and with_(_3=None) == INVALID and with_(_2=504) == INVALID
    assert with_(_6=132) == INVALID and with_(_8=9) == INVALID and with_(_10=4) == INVALID and with_(_12=0) == INVALID
    assert with_(_8=18, _2=2000) == UNSUPPORTED
    assert with_(_9=FAKE, _10=0) == 0  # nothing to append
    assert with_(_0=cache(pced, key_step=None)) == INVALID
    f = pced.lib().pced_paged_attention8
    good = [cache(pced), FAKE, 512, 8, None, 0, 0, 0.1, FAKE, 0, FAKE, FAKE, 1 << 30, None]
    assert with_(_1=None) == INVALID and with_(_2=100) == INVALID and with_(_5=3) == INVALID and with_(_6=-1) == INVALID
    assert with_(_7=float("nan")) == INVALID and with_(_8=FAKE + 4) == INVALID and with_(_9=2) == INVALID
    assert with_(_11=FAKE + 16) == WORKSPACE and with_(_12=16) == WORKSPACE
    assert with_(_3=18, _2=4096) == UNSUPPORTED


def test_sample_arguments(pced):
    f = pced.lib().pced_sample
    good = dict(x=FAKE, type=0, stride=100, rows=2, V=100, u=FAKE, t=FAKE, k=FAKE, p=FAKE, low=FAKE, token=FAKE, lp=FAKE,
                status=FAKE, stream=None)
    for kw in (dict(x=None), dict(u=None), dict(token=None), dict(type=2), dict(type=-1), dict(stride=99), dict(V=0),
               dict(rows=-1), dict(x=FAKE + 2), dict(x=FAKE + 1, type=1), dict(u=FAKE + 2), dict(t=FAKE + 1),
               dict(k=FAKE + 2), dict(p=FAKE + 3), dict(low=FAKE + 2), dict(token=FAKE + 2), dict(lp=FAKE + 2),
               dict(status=FAKE + 1)):
        assert f(*dict(good, **kw).values()) == INVALID, kw
    assert f(*dict(good, V=393_217, stride=1 << 20).values()) == UNSUPPORTED
    assert f(*dict(good, rows=1 << 30).values()) == UNSUPPORTED
    assert f(*dict(good, rows=0, x=None).values()) == 0


def make(pced, **kw):
    k = torch.zeros((4, 2, 16, 64), dtype=f8)
    return pced.PagedCache8(k, k.clone(), torch.ones((4, 2, 2)), torch.zeros((3, 2), dtype=i32),
                            torch.ones(3, dtype=i32), **kw)


def test_what_a_cache_is_made_of(pced):
    k, s = torch.zeros((4, 2, 16, 64), dtype=f8), torch.ones((4, 2, 2))
    table, lens = torch.zeros((3, 2), dtype=i32), torch.ones(3, dtype=i32)
    for args in ((k.float(), k, s, table, lens), (k, k.view(torch.uint8), s, table, lens), (None, k, s, table, lens),
                 (k, None, s, table, lens), (k, k, None, table, lens), (k, k, s.double(), table, lens),
                 (k, k, s[:3], table, lens), (k, k, s[..., :1], table, lens), (k, k, s.transpose(0, 1), table, lens),
                 (k, k, s, table.long(), lens), (k, k, s, table, lens[:2]), (k.to(bf), k.to(bf), s, table, lens),
                 (k.view(torch.float8_e5m2), k, s, table, lens)):
        with pytest.raises(ValueError):
            pced.PagedCache8(*args)
            pytest.fail("accepted")
    with pytest.raises(ValueError):  # e4m3 numbers without scales
        pced.PagedCache(k, k, table, lens)


@pytest.mark.parametrize("name", ["k", "v", "scale", "block_table", "seq_len"])
def test_other_tensors_are_refused(pced, name):
    c = make(pced)
    held = getattr(c, name)
    with pytest.raises(AttributeError, match=name):
        setattr(c, name, held.clone())
    at = c.struct8.scale if name == "scale" else getattr(c.struct8.pages, name)
    assert at == held.data_ptr() and c.at == ctypes.addressof(c.struct8)


def test_binding_refuses_bad_tensors(pced):
    c = make(pced, summary=torch.zeros((4, 2, 2, 64), dtype=torch.int8), key_step=torch.ones(2))
    q, kv = torch.zeros((3, 8, 64), dtype=bf), torch.zeros((3, 2, 64), dtype=bf)
    x, u = torch.zeros((4, 8)), torch.zeros(4)
    bad = [lambda: pced.kv_append(c, q, kv.to(f8), kv), lambda: pced.kv_append(c, q, kv[:, :1], kv),
           lambda: pced.kv_append(c, q[:2], kv, kv), lambda: pced.paged_attention(c, q[:2]),
           lambda: pced.paged_attention(c, q, out=q.double()),
           lambda: pced.paged_attention(c, q, sel=torch.zeros((3, 2, 0), dtype=i32)),
           lambda: pced.block_summaries(c),  # it reads bf16 keys
           lambda: pced.sample(x.double(), u), lambda: pced.sample(x.half(), u), lambda: pced.sample(x[0], u),
           lambda: pced.sample(x.t(), u), lambda: pced.sample(x, u[:3]), lambda: pced.sample(x, u.double()),
           lambda: pced.sample(x[:, :0], u), lambda: pced.sample(x, None),
           lambda: pced.sample(x, u, temperature=torch.ones(3)), lambda: pced.sample(x, u, temperature=1.0),
           lambda: pced.sample(x, u, top_k=torch.ones(4)), lambda: pced.sample(x, u, top_p=torch.ones(4, dtype=i32)),
           lambda: pced.sample(x, u, min_p=torch.ones(8)[::2]), lambda: pced.sample(x, u, token=torch.zeros(4)),
           lambda: pced.sample(x, u, logprob=torch.zeros(5)),
           lambda: pced.sample(x, u, status=torch.zeros(0, dtype=i32))]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {i} was accepted")


def test_binding_refuses_tensors_off_the_gpu(pced):
    c = make(pced)
    q, kv = torch.zeros((3, 8, 64), dtype=bf), torch.zeros((3, 2, 64), dtype=bf)
    for call in (lambda: pced.kv_append(c, q, kv, kv), lambda: pced.paged_attention(c, q, ws=torch.zeros(1 << 22, dtype=torch.uint8)),
                 lambda: pced.sample(torch.zeros(4, 8), torch.zeros(4))):
        with pytest.raises(ValueError, match="CUDA"):
            call()


def test_exports_and_loads(pced):
    # the declared functions whose names end in a digit, and the new one
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "pced.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(pced_[a-z_]+8)\s*\(", src)) | {"pced_sample"}
    assert {"pced_kv_append8", "pced_paged_attention8"} <= names
    for n in names:
        assert hasattr(pced.lib(), n), n


def test_no_non_coherent_reads_in_headers_and_new_kernels():
    # kernels launched programmatically read what an earlier launch writes with plain loads
    csrc = os.path.join(ROOT, "paper_2601_08670_gb300", "csrc")
    for path in glob.glob(os.path.join(csrc, "*.cuh")) + [os.path.join(csrc, f) for f in (
            "kv_append8.cu", "paged_attention8.cu", "sample.cu")]:
        src = re.sub(r"//[^\n]*", "", open(path).read())
        if "pdl_wait()" in src and "common.cuh" not in path:
            assert "__restrict__" not in src and "__ldg(" not in src and "ld.global.nc" not in src, path
