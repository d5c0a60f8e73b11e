"""GB300 (sm_103a) decode step of Parallel Context-of-Experts Decoding.

Thin binding of ``libpced.so`` (C ABI declared in ``include/pced.h``), through
ctypes, and for the calls over paged caches and on logits through a small
CPython module beside it (``pced_calls.so``): argument marshalling only, every
step of the computation runs in the library's CUDA kernels.  PyTorch supplies
device memory and streams.  There is no CPU fallback: if the library is not
built, every call raises.
"""
from __future__ import annotations

import ctypes
import importlib.machinery
import importlib.util
import math
import os

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
# PCED_LIB=checked selects the bounds-checked build (build.build(checked=True))
LIB_PATH = os.path.join(HERE, "_lib_checked" if os.environ.get("PCED_LIB") == "checked" else "_lib", "libpced.so")

PCED_DEV_BAD_LENGTH = 0x1
PCED_DEV_CACHE_FULL = 0x2
PCED_DEV_TIMEOUT = 0x4
PCED_DEV_BAD_TOKEN = 0x8
PCED_DEV_STEP_LIMIT = 0x10
PCED_DEV_BAD_BLOCK = 0x20
PCED_DEV_BOUNDS = 0x40
PCED_DEV_BAD_INDEX = 0x80
PCED_DEV_BAD_PARAM = 0x100


class PcedError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(msg)
        self.status = status


class Dims(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("N", ctypes.c_int32), ("L", ctypes.c_int32), ("Hq", ctypes.c_int32),
                ("Hkv", ctypes.c_int32), ("D", ctypes.c_int32), ("V", ctypes.c_int32)]


class StepArgs(ctypes.Structure):
    _fields_ = [("dims", Dims), ("embed", ctypes.c_void_p), ("w_unembed", ctypes.c_void_p),
                ("k_cache", ctypes.c_void_p), ("v_cache", ctypes.c_void_p), ("layer_elems", ctypes.c_int64),
                ("kv_offset", ctypes.c_void_p), ("cap", ctypes.c_void_p), ("total_cap", ctypes.c_int64),
                ("seq_len", ctypes.c_void_p), ("step", ctypes.c_void_p), ("history", ctypes.c_void_p),
                ("expert_trace", ctypes.c_void_p), ("score_trace", ctypes.c_void_p), ("gap_trace", ctypes.c_void_p),
                ("max_steps", ctypes.c_int32),
                ("beta", ctypes.c_void_p), ("r", ctypes.c_void_p), ("gamma", ctypes.c_float),
                ("attn_scale", ctypes.c_float), ("rms_eps", ctypes.c_float), ("bos_token", ctypes.c_int32),
                ("hidden_out", ctypes.c_void_p), ("lse_out", ctypes.c_void_p), ("workspace", ctypes.c_void_p),
                ("workspace_bytes", ctypes.c_size_t), ("stage_events", ctypes.c_void_p),
                ("n_stage_events", ctypes.c_int32), ("beta_from_step", ctypes.c_int32), ("beta_out", ctypes.c_void_p),
                ("block_table", ctypes.c_void_p), ("block_rows", ctypes.c_int32), ("max_blocks", ctypes.c_int32),
                ("rope_theta", ctypes.c_float), ("score_mode", ctypes.c_int32), ("aggregation", ctypes.c_int32),
                ("wait_limit_ns", ctypes.c_uint64), ("expert_base", ctypes.c_int32), ("key_out", ctypes.c_void_p),
                ("token_out", ctypes.c_void_p), ("expert_out", ctypes.c_void_p), ("score_out", ctypes.c_void_p)]


class PagedCacheStruct(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("summary", ctypes.c_void_p),
                ("key_step", ctypes.c_void_p), ("block_table", ctypes.c_void_p), ("seq_len", ctypes.c_void_p),
                ("num_blocks", ctypes.c_int32), ("block_rows", ctypes.c_int32), ("max_blocks", ctypes.c_int32),
                ("S", ctypes.c_int32), ("Hkv", ctypes.c_int32), ("D", ctypes.c_int32)]


class PagedCache8Struct(ctypes.Structure):
    _fields_ = [("pages", PagedCacheStruct), ("scale", ctypes.c_void_p)]


_lib = None


def lib(path: str = LIB_PATH):
    """Load libpced.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(path):
            raise RuntimeError(f"{path} is missing: build it with paper_2601_08670_gb300.build.build()")
        L = ctypes.CDLL(path)
        P, I32, I64, SZ, F = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t, ctypes.c_float
        L.pced_status_string.argtypes = [I32]
        L.pced_status_string.restype = ctypes.c_char_p
        L.pced_last_error.argtypes = []
        L.pced_last_error.restype = ctypes.c_char_p
        L.pced_decode_attention_workspace_size.argtypes = [I32, I32, I32, I32]
        L.pced_decode_attention_workspace_size.restype = SZ
        L.pced_decode_attention.argtypes = [P, P, P, I64, P, P, P, I32, I32, I32, I32, I64, F, P, P, SZ, P]
        L.pced_decode_attention.restype = I32
        L.pced_decode_attention_noalloc.argtypes = [P, P, P, I64, P, P, P, I32, I32, I32, I32, I64, F, P, P, P]
        L.pced_decode_attention_noalloc.restype = I32
        L.pced_lm_head_workspace_size.argtypes = [I32, I32]
        L.pced_lm_head_workspace_size.restype = SZ
        L.pced_lm_head_logprobs.argtypes = [P, P, I32, I32, I32, P, P, P, SZ, P]
        L.pced_lm_head_logprobs.restype = I32
        L.pced_contrastive_select_workspace_size.argtypes = [I32, I32, I32]
        L.pced_contrastive_select_workspace_size.restype = SZ
        L.pced_contrastive_select.argtypes = [P, P, P, F, I32, I32, I32, P, P, P, P, SZ, P]
        L.pced_contrastive_select.restype = I32
        L.pced_adacad_beta_workspace_size.argtypes = [I32, I32, I32]
        L.pced_adacad_beta_workspace_size.restype = SZ
        L.pced_adacad_beta.argtypes = [P, I32, I32, I32, P, P, SZ, P]
        L.pced_adacad_beta.restype = I32
        L.pced_relevance.argtypes = [P, I32, P, I32, ctypes.c_double, P, P]
        L.pced_relevance.restype = I32
        L.pced_step_workspace_size.argtypes = [ctypes.POINTER(Dims)]
        L.pced_step_workspace_size.restype = SZ
        L.pced_step.argtypes = [ctypes.POINTER(StepArgs), P]
        L.pced_step.restype = I32
        L.pced_step_host_io.argtypes = [ctypes.POINTER(StepArgs), P, P, P, P, P, P]
        L.pced_step_host_io.restype = I32
        L.pced_step_launch_count.argtypes = [ctypes.POINTER(StepArgs)]
        L.pced_step_launch_count.restype = I32
        L.pced_step_launch_kind.argtypes = [ctypes.POINTER(StepArgs), I32]
        L.pced_step_launch_kind.restype = ctypes.c_char_p
        L.pced_select_key.argtypes = [F, I32, I32]
        L.pced_select_key.restype = I64
        L.pced_select_key_unpack.argtypes = [I64, ctypes.POINTER(F), ctypes.POINTER(I32), ctypes.POINTER(I32)]
        L.pced_select_key_unpack.restype = None
        L.pced_step_commit.argtypes = [P, I32, P, P, P, P, I32, P, P]
        L.pced_step_commit.restype = I32
        C = ctypes.POINTER(PagedCacheStruct)
        L.pced_kv_append.argtypes = [C, P, I64, P, I64, P, I64, P, I32, P, I32, P, I32, P, P, P]
        L.pced_kv_append.restype = I32
        L.pced_block_summaries.argtypes = [C, P, P]
        L.pced_block_summaries.restype = I32
        L.pced_block_select.argtypes = [C, P, I64, I32, I32, I32, I32, P, P, P]
        L.pced_block_select.restype = I32
        L.pced_paged_attention_workspace_size.argtypes = [I32, I32, I32, I32]
        L.pced_paged_attention_workspace_size.restype = SZ
        L.pced_paged_attention.argtypes = [C, P, I64, I32, P, I32, I64, F, P, I32, P, P, SZ, P]
        L.pced_paged_attention.restype = I32
        L.pced_logits_process.argtypes = [P, P, I64, I32, I32, I32, P, I32, P, P, P, P, I32, P, I32, I32, P, P, P]
        L.pced_logits_process.restype = I32
        C8 = ctypes.POINTER(PagedCache8Struct)
        L.pced_kv_append8.argtypes = [C8, *L.pced_kv_append.argtypes[1:]]
        L.pced_kv_append8.restype = I32
        L.pced_paged_attention8.argtypes = [C8, *L.pced_paged_attention.argtypes[1:]]
        L.pced_paged_attention8.restype = I32
        L.pced_sample.argtypes = [P, I32, I64, I32, I32, P, P, P, P, P, P, P, P, P]
        L.pced_sample.restype = I32
        _lib = L
    return _lib


_calls = None


def _native():
    """The CPython module of the calls over paged caches and on logits (raises if it has not been built)."""
    global _calls
    if _calls is None:
        lib()
        path = os.path.join(os.path.dirname(LIB_PATH), "pced_calls.so")
        if not os.path.exists(path):
            raise RuntimeError(f"{path} is missing: build it with paper_2601_08670_gb300.build.build()")
        loader = importlib.machinery.ExtensionFileLoader("pced_calls", path)
        module = importlib.util.module_from_spec(importlib.util.spec_from_loader("pced_calls", loader))
        loader.exec_module(module)
        _calls = module
    return _calls


def _check(rc: int, what: str):
    if rc != 0:
        L = lib()
        raise PcedError(rc, f"{what}: {L.pced_status_string(rc).decode()}: {L.pced_last_error().decode()}")


def _require(cond: bool, what: str):
    """Argument check of the binding (raises even under python -O)."""
    if not cond:
        raise ValueError(what)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream(stream=None):
    """The raw handle of `stream`, by default of the current stream (asked for
    directly: building the torch.cuda.Stream object costs 3 us per call, a
    quarter of what a small call takes on the host)."""
    if stream is not None:
        return stream.cuda_stream
    if not torch.cuda.is_initialized():
        torch.cuda.init()
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def workspace(nbytes: int, device) -> torch.Tensor:
    """Zeroed workspace (the device status word at byte 0 starts clear)."""
    return torch.zeros(max(int(nbytes), 256), dtype=torch.uint8, device=device)


def device_status(ws: torch.Tensor) -> int:
    """Device status bits the kernels ORed into the workspace (synchronises)."""
    return int(ws[:4].view(torch.int32).item())


# ------------------------------------------------------------------ entry points
def decode_attention_workspace_size(S, Hq, Hkv, D) -> int:
    return int(lib().pced_decode_attention_workspace_size(S, Hq, Hkv, D))


def decode_attention(q, k_cache, v_cache, kv_offset, cap, seq_len, Hkv: int, total_cap: int, scale=None, out=None,
                     ws=None, stream=None):
    """pced_decode_attention: q bf16 [S, Hq, D]; caches bf16 (one layer); returns fp32 [S, Hq, D]."""
    S, Hq, D = q.shape
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    if out is None:
        out = torch.empty((S, Hq, D), dtype=torch.float32, device=q.device)
    if ws is None:
        ws = workspace(decode_attention_workspace_size(S, Hq, Hkv, D), q.device)
    _check(lib().pced_decode_attention(_ptr(q), _ptr(k_cache), _ptr(v_cache), k_cache.numel(), _ptr(kv_offset),
                                       _ptr(cap), _ptr(seq_len), S, Hq, Hkv, D, int(total_cap), float(scale),
                                       _ptr(out), _ptr(ws), ws.numel(), _stream(stream)), "pced_decode_attention")
    return out


# fixed size of the library's scratch array behind decode_attention_noalloc
NOALLOC_SCRATCH_BYTES = 16 << 20


def decode_attention_noalloc(q, k_cache, v_cache, kv_offset, cap, seq_len, Hkv: int, total_cap: int, out,
                             scale=None, status=None, stream=None):
    """pced_decode_attention_noalloc: decode_attention without a workspace.

    For callers that cannot allocate device memory when they run attention
    (allocator locked or shutting down, host callbacks, capped memory pools):
    the partial records live in a fixed library-owned device array, so the
    caller passes the output buffer ``out`` (fp32 [S, Hq, D]) and, optionally,
    an int32 device ``status`` word.  Calls share that array: overlapping calls
    on the GPU race.  The first call on a device should come before any stream
    capture on it."""
    S, Hq, D = q.shape
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    _check(lib().pced_decode_attention_noalloc(_ptr(q), _ptr(k_cache), _ptr(v_cache), k_cache.numel(),
                                               _ptr(kv_offset), _ptr(cap), _ptr(seq_len), S, Hq, Hkv, D,
                                               int(total_cap), float(scale), _ptr(out),
                                               None if status is None else _ptr(status), _stream(stream)),
           "pced_decode_attention_noalloc")
    return out


def lm_head_workspace_size(S, V) -> int:
    return int(lib().pced_lm_head_workspace_size(S, V))


def lm_head_logprobs(hidden, w_unembed, logprobs=None, lse=None, ws=None, stream=None):
    """pced_lm_head_logprobs: hidden bf16 [S, d], W bf16 [V, d] -> (fp32 [S, V], fp32 [S])."""
    S, d = hidden.shape
    V = w_unembed.shape[0]
    if logprobs is None:
        logprobs = torch.empty((S, V), dtype=torch.float32, device=hidden.device)
    if lse is None:
        lse = torch.empty(S, dtype=torch.float32, device=hidden.device)
    if ws is None:
        ws = workspace(lm_head_workspace_size(S, V), hidden.device)
    _check(lib().pced_lm_head_logprobs(_ptr(hidden), _ptr(w_unembed), S, d, V, _ptr(logprobs), _ptr(lse), _ptr(ws),
                                       ws.numel(), _stream(stream)), "pced_lm_head_logprobs")
    return logprobs, lse


def contrastive_select_workspace_size(B, N, V) -> int:
    return int(lib().pced_contrastive_select_workspace_size(B, N, V))


def contrastive_select(logprobs, beta, r, gamma: float, ws=None, stream=None):
    """pced_contrastive_select: returns (token [B] int32, expert [B] int32, score [B] fp32)."""
    B, N = beta.shape
    V = logprobs.shape[1]
    dev = logprobs.device
    token = torch.empty(B, dtype=torch.int32, device=dev)
    expert = torch.empty(B, dtype=torch.int32, device=dev)
    score = torch.empty(B, dtype=torch.float32, device=dev)
    if ws is None:
        ws = workspace(contrastive_select_workspace_size(B, N, V), dev)
    _check(lib().pced_contrastive_select(_ptr(logprobs), _ptr(beta), _ptr(r), float(gamma), B, N, V, _ptr(token),
                                         _ptr(expert), _ptr(score), _ptr(ws), ws.numel(), _stream(stream)),
           "pced_contrastive_select")
    return token, expert, score


def adacad_beta(logprobs, B: int, N: int, ws=None, stream=None):
    """pced_adacad_beta: per-expert Jensen-Shannon divergence (bits) between
    each expert's distribution and its query's amateur, fp32 [B, N]."""
    V = logprobs.shape[1]
    beta = torch.empty((B, N), dtype=torch.float32, device=logprobs.device)
    if ws is None:
        ws = workspace(int(lib().pced_adacad_beta_workspace_size(B, N, V)), logprobs.device)
    _check(lib().pced_adacad_beta(_ptr(logprobs), B, N, V, _ptr(beta), _ptr(ws), ws.numel(), _stream(stream)),
           "pced_adacad_beta")
    return beta


RET_DENSE, RET_SPARSE = 0, 1
SCORE_LOGPROB, SCORE_LOGIT = 0, 1
AGG_MAX, AGG_MOE, AGG_POE = 0, 1, 2


def relevance(ret_scores, ret_mode: int = RET_DENSE, rer_logits=None, eps: float = 1e-8, stream=None):
    """pced_relevance: relevance scores in [0, 1) from raw retrieval scores
    (dense/ColBERT or sparse) and optional reranker logits, fused by the
    harmonic mean (fp32 tensors of one shape on the device)."""
    _require(ret_scores.dtype == torch.float32 and ret_scores.is_contiguous(), "ret_scores: contiguous fp32")
    if rer_logits is not None:
        _require(rer_logits.dtype == torch.float32 and rer_logits.is_contiguous(), "rer_logits: contiguous fp32")
        _require(rer_logits.shape == ret_scores.shape, "rer_logits: the shape of ret_scores")
    r = torch.empty_like(ret_scores)
    _check(lib().pced_relevance(_ptr(ret_scores), int(ret_mode), _ptr(rer_logits), ret_scores.numel(), float(eps),
                                _ptr(r), _stream(stream)), "pced_relevance")
    return r


# ------------------------------------------- operators over paged caches
def _empty(shape, dtype, device, stream):
    """torch.empty in the memory of the stream that will write it."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _is(t, dtype, shape):
    return t.dtype == dtype and t.shape == shape and t.is_contiguous()


def _handle(stream, gpu):
    """The raw handle of a stream of device `gpu`."""
    _require(getattr(stream, "device_index", gpu) == gpu, "the stream is another device's than the tensors")
    return stream.cuda_stream


class PagedCache:
    """One layer's paged cache of S sequences (pced_paged_cache in pced.h):

    ``k``, ``v``       bf16 [num_blocks, Hkv, block_rows, D], the layout of pced_step's paged caches
    ``block_table``    int32 [S, max_blocks]
    ``seq_len``        int32 [S]: live rows, the rows appended in this step included
    ``summary``        int8 [num_blocks, Hkv, 2, D] and
    ``key_step``       fp32 [Hkv]: the blocks' key summaries, for block_select (optional)

    k and v may be None where only block_select is called (block_rows is then needed).  The tensors are held,
    and their addresses taken once: change their contents, not their storage (the fields take no other tensor; for
    one, make another PagedCache).  They lie on one CUDA device, which is the current one when the calls are made."""

    _TAKEN = frozenset(["k", "v", "block_table", "seq_len", "summary", "key_step", "num_blocks", "Hkv", "block_rows",
                        "D", "S", "max_blocks"])
    _NUMBERS, _NAME = torch.bfloat16, "bf16"
    eight = False  # whether k and v are 8-bit numbers with scales

    def __setattr__(self, name, value):
        # (`cache.seq_len += 1` works in place and puts the same tensor back)
        if name in self._TAKEN and self.__dict__.get(name, value) is not value:
            raise AttributeError(f"{name}: its address or size has been taken; make another PagedCache")
        super().__setattr__(name, value)

    def __delattr__(self, name):
        if name in self._TAKEN:
            raise AttributeError(f"{name}: its address or size has been taken")
        super().__delattr__(name)

    def __init__(self, k, v, block_table, seq_len, *, block_rows=None, summary=None, key_step=None):
        _require(k is not None or (summary is not None and block_rows is not None),
                 "k, or a summary and block_rows, are needed")
        if k is not None:
            _require(k.dim() == 4, "k: [num_blocks, Hkv, block_rows, D]")
            nb, Hkv, P, D = k.shape
            _require(block_rows is None or block_rows == P, "block_rows differs from k's")
        else:
            _require(summary.dim() == 4, "summary: [num_blocks, Hkv, 2, D]")
            nb, Hkv, P, D = summary.shape[0], summary.shape[1], int(block_rows), summary.shape[3]
        for name, t in (("k", k), ("v", v)):
            _require(t is None or _is(t, self._NUMBERS, (nb, Hkv, P, D)),
                     f"{name}: contiguous {self._NAME} [num_blocks, Hkv, block_rows, D]")
        _require(summary is None or _is(summary, torch.int8, (nb, Hkv, 2, D)),
                 "summary: contiguous int8 [num_blocks, Hkv, 2, D]")
        _require(key_step is None or _is(key_step, torch.float32, (Hkv,)), "key_step: fp32 [Hkv]")
        _require(block_table.dim() == 2 and block_table.dtype == torch.int32 and block_table.is_contiguous(),
                 "block_table: contiguous int32 [S, max_blocks]")
        S = block_table.shape[0]
        _require(_is(seq_len, torch.int32, (S,)), "seq_len: contiguous int32 [S]")
        self.k, self.v, self.block_table, self.seq_len, self.summary, self.key_step = (k, v, block_table, seq_len,
                                                                                       summary, key_step)
        self.num_blocks, self.Hkv, self.block_rows, self.D, self.S = nb, Hkv, P, D, S
        self.max_blocks = block_table.shape[1]
        self.device = block_table.device
        for t in (k, v, seq_len, summary, key_step):
            _require(t is None or t.device == self.device, "a cache's tensors lie on one device")
        self.struct = PagedCacheStruct(_ptr(k), _ptr(v), _ptr(summary), _ptr(key_step), _ptr(block_table),
                                       _ptr(seq_len), nb, P, self.max_blocks, S, Hkv, D)
        self.at = ctypes.addressof(self.struct)
        self.gpu = self.device.index if self.device.type == "cuda" else -1


class PagedCache8(PagedCache):
    """One layer's paged cache in 8 bits (pced_paged_cache8 in pced.h), for the same calls as a PagedCache:

    ``k``, ``v``       e4m3 (torch.float8_e4m3fn) [num_blocks, Hkv, block_rows, D]
    ``scale``          fp32 [num_blocks, Hkv, 2]: what a block's numbers are multiples of, keys' and values'
    and the other tensors of a PagedCache.

    kv_append writes numbers and scales (rows of another cache become bytes by appending them), paged_attention reads
    them, block_select reads the summaries, which kv_append keeps; block_summaries reads bf16 keys and takes a
    PagedCache alone."""

    _TAKEN = PagedCache._TAKEN | {"scale"}
    _NUMBERS, _NAME = torch.float8_e4m3fn, "e4m3"
    eight = True

    def __init__(self, k, v, scale, block_table, seq_len, *, summary=None, key_step=None):
        _require(k is not None and v is not None and scale is not None, "k, v and scale are needed")
        super().__init__(k, v, block_table, seq_len, summary=summary, key_step=key_step)
        _require(_is(scale, torch.float32, (self.num_blocks, self.Hkv, 2)),
                 "scale: contiguous fp32 [num_blocks, Hkv, 2]")
        _require(scale.device == self.device, "a cache's tensors lie on one device")
        self.scale = scale
        self.struct8 = PagedCache8Struct(self.struct, _ptr(scale))
        self.struct = self.struct8.pages
        self.at = ctypes.addressof(self.struct8)


def rope_table(theta: float, D: int, rows: int, device="cuda") -> torch.Tensor:
    """Rotation table of kv_append, fp32 [rows, D]: cosines, then sines, of the
    angles fp32(p * fp32(theta^(-2f/D))), which pced_step rotates by."""
    f = torch.tensor([theta ** (-2.0 * i / D) for i in range(D // 2)], dtype=torch.float32, device=device)
    angle = (torch.arange(rows, dtype=torch.float32, device=device)[:, None] * f).double()
    return torch.cat([angle.cos(), angle.sin()], dim=1).float()


def kv_append(cache: PagedCache, q, k, v, rope=None, tok_start=None, positions=None, q_out=None, status=None,
              stream=None):
    """pced_kv_append (pced_kv_append8 for a PagedCache8): k, v bf16 [T, Hkv, D] into the last rows of the sequences,
    q bf16 [T, Hq, D] (or None) rotated into q_out, which is returned.  The parts of one projection's output need no
    copies (strides between tokens).  rope: fp32 [rows, D] (rope_table), None: no rotation; tok_start: int32 [S + 1],
    None: one token per sequence; positions: int32 [T], None: the rows themselves.  Device conditions go to the int32
    tensor status."""
    if q_out is None and q is not None:
        q_out = _empty((q.shape[0], q.shape[1], cache.D), torch.bfloat16, q.device, stream)
    native = _calls or _native()
    rc = (native.kv_append8 if cache.eight else native.kv_append)(
        cache.at, cache.gpu, q, k, v, rope, tok_start, positions, q_out, status,
        None if stream is None else _handle(stream, cache.gpu))
    if rc:
        _check(rc, "pced_kv_append8" if cache.eight else "pced_kv_append")
    return q_out


def block_summaries(cache: PagedCache, status=None, stream=None):
    """pced_block_summaries: cache.summary from the cached keys of all live blocks; returns it."""
    _require(not cache.eight, "block_summaries reads bf16 keys; kv_append keeps the summaries of a PagedCache8")
    rc = (_calls or _native()).block_summaries(cache.at, cache.gpu, status,
                                               None if stream is None else _handle(stream, cache.gpu))
    if rc:
        _check(rc, "pced_block_summaries")
    return cache.summary


def block_select(cache: PagedCache, q, n_sel: int, n_first: int = 1, n_last: int = 1, sel=None, status=None,
                 stream=None):
    """pced_block_select: int32 [S, Hkv, n_sel], the blocks that q bf16 [S, Hq, D] attends to in ascending order
    (-1 after the last): the first n_first, the last n_last and those with the highest scores."""
    if sel is None:
        sel = _empty((cache.S, cache.Hkv, n_sel), torch.int32, q.device, stream)
    rc = (_calls or _native()).block_select(cache.at, cache.gpu, q, n_sel, n_first, n_last, sel, status,
                                            None if stream is None else _handle(stream, cache.gpu))
    if rc:
        _check(rc, "pced_block_select")
    return sel


def paged_attention_workspace_size(S, Hq, Hkv, D) -> int:
    return int(lib().pced_paged_attention_workspace_size(S, Hq, Hkv, D))


def paged_attention(cache: PagedCache, q, sel=None, total_rows: int = 0, scale=None, out=None, lse=None, ws=None,
                    stream=None):
    """pced_paged_attention (pced_paged_attention8 for a PagedCache8): q bf16 [S, Hq, D] over the cache, or over the
    blocks sel int32 [S, Hkv, n_sel]; returns out [S, Hq, D], fp32 unless a bf16 `out` is passed.  lse: fp32 [S, Hq]
    that receives the log of the softmax's sum.  total_rows: upper bound of the rows attended to (of one kv-head, over
    all sequences), 0: unknown.  A workspace of the caller's own is zeroed before its first use (workspace())."""
    if out is None:
        out = _empty((cache.S, q.shape[1], cache.D), torch.float32, q.device, stream)
    if ws is None:
        ws = _empty(max(256, paged_attention_workspace_size(cache.S, q.shape[1], cache.Hkv, cache.D)), torch.uint8,
                    q.device, stream)
        with torch.cuda.stream(stream):  # (None: the current one)
            ws.zero_()
    native = _calls or _native()
    rc = (native.paged_attention8 if cache.eight else native.paged_attention)(
        cache.at, cache.gpu, q, sel, total_rows, 1.0 / math.sqrt(cache.D) if scale is None else scale, out, lse, ws,
        None if stream is None else _handle(stream, cache.gpu))
    if rc:
        _check(rc, "pced_paged_attention8" if cache.eight else "pced_paged_attention")
    return out


def logits_process(logits, rows_per_query: int, history=None, history_len=None, penalties=None, bias_ids=None,
                   bias=None, mask=None, mask_row=None, out=None, status=None, stream=None):
    """pced_logits_process: logits fp32 [B * rows_per_query, V] (rows may be strided) with the penalties of repeated
    tokens (history int32 [B, n], history_len int32 [B], penalties fp32 [B, 3]: repetition, frequency, presence),
    biases (bias_ids int32 and bias fp32 [B, n]) and masks (int32 words [n_masks, ceil(V / 32)], bit set: allowed;
    mask_row int32 [B], -1: none) applied; normalise them afterwards.  out: another buffer of that shape and stride,
    or logits itself (in place); returned."""
    if out is None:
        rows, V = logits.shape
        out = _empty((rows, logits.stride(0) if rows > 1 else V), torch.float32, logits.device, stream)[:, :V]
    rc = (_calls or _native()).logits_process(logits, rows_per_query, history, history_len, penalties, bias_ids, bias,
                                              mask, mask_row, out, status,
                                              None if stream is None else _handle(stream, logits.get_device()))
    if rc:
        _check(rc, "pced_logits_process")
    return out


def sample(logits, u, temperature=None, top_k=None, top_p=None, min_p=None, token=None, logprob=None, status=None,
           stream=None):
    """pced_sample: int32 [rows], a token for every row of logits fp32 or bf16 [rows, V] (rows may be strided), drawn by
    u fp32 [rows] in [0, 1].  temperature, top_p, min_p fp32 [rows] and top_k int32 [rows]: each row's own (None: 1,
    and no cut).  logprob: fp32 [rows] that receives the tokens' log-probabilities under what they were drawn from.  A
    row without a token that could be drawn gets -1."""
    if token is None:
        token = _empty((logits.shape[0],), torch.int32, logits.device, stream)
    rc = (_calls or _native()).sample(logits, u, temperature, top_k, top_p, min_p, token, logprob, status,
                                      None if stream is None else _handle(stream, logits.get_device()))
    if rc:
        _check(rc, "pced_sample")
    return token


def dims(B, N, L, Hq, Hkv, D, V) -> Dims:
    return Dims(B, N, L, Hq, Hkv, D, V)


def step_workspace_size(dm: Dims) -> int:
    return int(lib().pced_step_workspace_size(ctypes.byref(dm)))


def step_launch_count(args) -> int:
    """Kernel launches of one pced_step call with these StepArgs."""
    return int(lib().pced_step_launch_count(ctypes.byref(args)))


def select_key(score: float, token: int, expert: int) -> int:
    """Eq. 3's choice as an int64 whose signed order is Eq. 3's order
    (pced_select_key)."""
    return int(lib().pced_select_key(float(score), int(token), int(expert)))


def select_key_unpack(key: int):
    """(fp32 score, token, expert) of a packed key."""
    s, t, e = ctypes.c_float(), ctypes.c_int32(), ctypes.c_int32()
    lib().pced_select_key_unpack(int(key), ctypes.byref(s), ctypes.byref(t), ctypes.byref(e))
    return s.value, t.value, e.value


def step_launch_kinds(args) -> list:
    return [lib().pced_step_launch_kind(ctypes.byref(args), i).decode() for i in range(step_launch_count(args))]


class Decoder:
    """Device-resident PCED decoding state and the pced_step call.

    Holds references to the caller's caches and weights, and owns the step
    counter, the generated history, the expert trace and the workspace.  Each
    ``step()`` is one pced_step call (asynchronous on the current stream)."""

    def __init__(self, dm: Dims, *, embed, w_unembed, k_cache, v_cache, layer_elems: int, kv_offset, cap, seq_len,
                 beta, r, gamma: float, max_steps: int, total_cap: int, bos: int = 0, attn_scale=None,
                 rms_eps: float = 1e-6, keep_hidden: bool = False, dynamic_beta: bool = False, block_table=None,
                 block_rows: int = 0, rope_theta: float = 0.0, score_mode: int = 0, aggregation: int = 0,
                 track_gaps: bool = True):
        dev = k_cache.device
        self.dm = dm
        B, S, d = dm.B, dm.B * (dm.N + 1), dm.Hq * dm.D
        self.step_t = torch.zeros(1, dtype=torch.int32, device=dev)
        self.history = torch.zeros((B, max_steps), dtype=torch.int32, device=dev)
        self.expert_trace = torch.zeros((B, max_steps), dtype=torch.int32, device=dev)
        self.score_trace = torch.zeros((B, max_steps), dtype=torch.float32, device=dev)
        # near-tie margins of every choice: [B, max_steps, 2] (token gap, expert gap)
        self.gap_trace = torch.zeros((B, max_steps, 2), dtype=torch.float32, device=dev) if track_gaps else None
        # this step's choice at fixed addresses (the traces move with t)
        # (one [3, B] block, so that reading all three back is one copy)
        self._choice = torch.zeros((3, B), dtype=torch.int32, device=dev)
        self.token_out, self.expert_out = self._choice[0], self._choice[1]
        self.score_out = self._choice[2].view(torch.float32)
        self.hidden = torch.zeros((S, d), dtype=torch.bfloat16, device=dev) if keep_hidden else None
        self.lse = torch.zeros(S, dtype=torch.float32, device=dev)
        self.ws = workspace(step_workspace_size(dm), dev)
        self._keep = (embed, w_unembed, k_cache, v_cache, kv_offset, cap, seq_len, beta, r, block_table)
        self.seq_len = seq_len
        self.beta, self.r = beta, r
        self.args = StepArgs(
            dm, _ptr(embed), _ptr(w_unembed), _ptr(k_cache), _ptr(v_cache), int(layer_elems), _ptr(kv_offset),
            _ptr(cap), int(total_cap), _ptr(seq_len), _ptr(self.step_t), _ptr(self.history),
            _ptr(self.expert_trace), _ptr(self.score_trace), _ptr(self.gap_trace), int(max_steps), _ptr(beta), _ptr(r),
            float(gamma),
            float(1.0 / math.sqrt(dm.D) if attn_scale is None else attn_scale), float(rms_eps), int(bos),
            _ptr(self.hidden), _ptr(self.lse), _ptr(self.ws), self.ws.numel())
        self.max_steps = max_steps
        self.args.token_out = _ptr(self.token_out)
        self.args.expert_out = _ptr(self.expert_out)
        self.args.score_out = _ptr(self.score_out)
        self.args.rope_theta = float(rope_theta)  # rotary base, 0: none
        self.args.score_mode = int(score_mode)     # SCORE_LOGPROB / SCORE_LOGIT
        self.args.aggregation = int(aggregation)   # AGG_MAX / AGG_MOE / AGG_POE
        if block_table is not None:  # paged caches
            _require(block_table.dtype == torch.int32 and block_table.is_contiguous() and block_table.dim() == 2,
                     "block_table: contiguous int32 [S, max_blocks]")
            self.args.block_table = _ptr(block_table)
            self.args.block_rows = int(block_rows)
            self.args.max_blocks = int(block_table.shape[1])
        # dynamic contrast strength: the first step computes beta (into the
        # `beta` tensor, which the later steps read) from its distributions
        if dynamic_beta:
            _require(beta.dtype == torch.float32 and beta.is_contiguous(),
                     "beta: contiguous fp32 (dynamic beta writes it)")
            self.args.beta_from_step = 1
            self.args.beta_out = _ptr(beta)

    def step(self, stream=None):
        _check(lib().pced_step(ctypes.byref(self.args), _stream(stream)), "pced_step")
        self.args.beta_from_step = 0

    def step_host_io(self, beta=None, r=None, token=None, expert=None, score=None, stream=None):
        """One step with host buffers (pced_step_host_io): uploads `beta` / `r`
        (host fp32 [B, N], None: keep the device values), steps, and copies
        the choice into `token` / `expert` / `score` (host [B] int32 / int32 /
        fp32, None: skip).  Asynchronous on the stream; use page-locked
        tensors (pin_memory()) for asynchronous copies and graph capture.
        Adjacent buffers on both sides (r right after beta; expert after
        token, score after expert, as choice_buffers() lays them out) move
        in one copy each way."""
        B, N = self.dm.B, self.dm.N

        def host(t, dtype, n):
            if t is None:
                return None
            _require(t.device.type == "cpu" and t.dtype == dtype and t.is_contiguous() and t.numel() == n,
                     f"host buffers: contiguous {dtype} CPU tensors of {n} elements")
            return t.data_ptr()

        _check(lib().pced_step_host_io(ctypes.byref(self.args), host(beta, torch.float32, B * N),
                                       host(r, torch.float32, B * N), host(token, torch.int32, B),
                                       host(expert, torch.int32, B), host(score, torch.float32, B),
                                       _stream(stream)), "pced_step_host_io")
        self.args.beta_from_step = 0

    def choice_buffers(self):
        """Page-locked host (token, expert, score) tensors laid out like the
        device outputs, so step_host_io reads them back in one copy."""
        blk = torch.zeros((3, self.dm.B), dtype=torch.int32).pin_memory()
        return blk[0], blk[1], blk[2].view(torch.float32)

    def capture_host_io(self, beta=None, r=None, token=None, expert=None, score=None):
        """A CUDA graph of one step_host_io call: each replay is one decode
        step with its uploads and read-backs (page-locked host tensors
        required; the decoder's dynamic-beta first step must already be done)."""
        _require(not self.args.beta_from_step, "run the dynamic-beta first step before capturing")
        for t in (beta, r, token, expert, score):
            _require(t is None or t.is_pinned(), "graph capture needs page-locked host tensors")
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            self.step_host_io(beta, r, token, expert, score)
        return g

    def step_partial(self, keys, expert_base: int, stream=None):
        """Expert-partitioned step: this decoder's experts are global experts
        expert_base + 1 .. expert_base + N; writes their best choice per query
        as packed keys (int64 [B] device tensor `keys`) and appends nothing.
        Reduce the keys with a max over the decoders (NCCL / gloo all-reduce,
        torch.maximum), then call commit()."""
        _require(keys.dtype == torch.int64 and keys.is_contiguous() and keys.numel() >= self.dm.B,
                 "keys: contiguous int64 of at least B elements")
        self.args.key_out = _ptr(keys)
        self.args.expert_base = int(expert_base)
        try:
            self.step(stream)
        finally:
            self.args.key_out = None
            self.args.expert_base = 0

    def commit(self, keys, stream=None):
        """Append the reduced choices (int64 [B] device keys) and advance t."""
        _check(lib().pced_step_commit(_ptr(keys), self.dm.B, _ptr(self.step_t), _ptr(self.history),
                                      _ptr(self.expert_trace), _ptr(self.score_trace), self.max_steps,
                                      _ptr(self.ws), _stream(stream)), "pced_step_commit")

    def set_stage_events(self, events):
        """Record one torch.cuda.Event before and after every launch of each
        subsequent step (None disables)."""
        if events is None:
            self._events = None
            self.args.stage_events = None
            self.args.n_stage_events = 0
            return
        for ev in events:  # torch creates the CUDA event on its first record
            if ev.cuda_event == 0:
                ev.record()
        torch.cuda.synchronize()
        self._events = events
        self._event_handles = (ctypes.c_void_p * len(events))(*[ev.cuda_event for ev in events])
        self.args.stage_events = ctypes.cast(self._event_handles, ctypes.c_void_p)
        self.args.n_stage_events = len(events)

    def launches_per_step(self) -> int:
        """Kernel launches of the next step() call."""
        return step_launch_count(self.args)

    def launch_kinds(self) -> list:
        return step_launch_kinds(self.args)

    def status(self) -> int:
        return device_status(self.ws)


def decoder_from_inputs(dm: Dims, t: dict, *, gamma: float, max_steps: int, bos: int = 0, keep_hidden=False,
                        attn_scale=None, rms_eps: float = 1e-6, dynamic_beta: bool = False,
                        rope_theta: float = 0.0, score_mode: int = 0, aggregation: int = 0,
                        track_gaps: bool = True) -> Decoder:
    """Decoder over a dict of device tensors with the keys k_cache, v_cache,
    kv_offset, cap, seq_len, embed, w_unembed, beta, r, and the host layout
    values layer_elems / total_cap (or a `layout` object carrying them)."""
    lay = t.get("layout")
    layer_elems = t["layer_elems"] if "layer_elems" in t else lay.layer_elems
    total_cap = t["total_cap"] if "total_cap" in t else int(lay.cap.astype("int64").sum())
    return Decoder(dm, embed=t["embed"], w_unembed=t["w_unembed"], k_cache=t["k_cache"], v_cache=t["v_cache"],
                   layer_elems=layer_elems, kv_offset=t["kv_offset"], cap=t["cap"], seq_len=t["seq_len"],
                   beta=t["beta"], r=t["r"], gamma=gamma, max_steps=max_steps, total_cap=total_cap, bos=bos,
                   attn_scale=attn_scale, rms_eps=rms_eps, keep_hidden=keep_hidden, dynamic_beta=dynamic_beta,
                   block_table=t.get("block_table"), block_rows=int(t.get("block_rows", 0)), rope_theta=rope_theta,
                   score_mode=score_mode, aggregation=aggregation, track_gaps=track_gaps)
