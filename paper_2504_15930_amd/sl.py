"""Binding of ``libsl`` (``include/sl.h``), by ctypes and, for the 4-bit cache and the page bookkeeping,
``csrc/binding.cpp``: argument marshalling only.

Every step of the decode path (KV append and attention) runs in the HIP kernels of
``libsl.so``; torch supplies device memory, the current stream and (for
profiling) events. There is no fallback: without the built library or
without a GPU tensor every entry point raises.
"""
from __future__ import annotations

import contextlib
import ctypes
import functools
import os
import threading
import warnings

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
# SL_LIBRARY may name another build of the same sources (the host-sanitized one of the tests).
LIBRARY = os.environ.get("SL_LIBRARY") or os.path.join(HERE, "libsl.so")

PAGE_SIZE = 16
SL_OK = 0
STATUS_NAMES = {0: "SL_OK", -1: "SL_ERR_NULL", -2: "SL_ERR_SHAPE", -3: "SL_ERR_UNSUPPORTED",
                -4: "SL_ERR_WORKSPACE", -5: "SL_ERR_HIP", -6: "SL_ERR_ALIGNMENT", -7: "SL_ERR_SCRATCH_LIMIT"}
EXPORTS = ["sl_decode_attn_workspace_size", "sl_decode_attn_num_workers", "sl_decode_attn",
           "sl_decode_attn_fp8", "sl_kv_append", "sl_kv_append_fp8", "sl_decode_attn_prefix",
           "sl_decode_attn_prefix_fp8", "sl_decode_attn_prefix_workspace_size", "sl_decode_attn_noalloc",
           "sl_decode_attn_fp4", "sl_decode_attn_prefix_fp4", "sl_kv_append_fp4", "sl_kv_write_fp4", "sl_kv_read_fp4",
           "sl_pages_extend", "sl_pages_release", "sl_status_string"]
# include/sl_engine.h (typed in engine.py)
ENGINE_EXPORTS = ["sl_engine_create", "sl_engine_run", "sl_engine_schedule", "sl_engine_destroy"]
# include/sl_dispatch.h (typed in dispatch.py)
DISPATCH_EXPORTS = ["sl_generation_latency", "sl_dispatch_plan"]


class SlError(RuntimeError):
    """A libsl call returned an error status."""

    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {STATUS_NAMES.get(status, status)} ({status_string(status)})")


class Desc(ctypes.Structure):
    """Mirror of ``sl_attn_desc``."""

    _fields_ = [
        ("batch", ctypes.c_int32),
        ("num_q_heads", ctypes.c_int32),
        ("num_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("page_size", ctypes.c_int32),
        ("max_blocks_per_seq", ctypes.c_int32),
        ("num_pages", ctypes.c_int32),
        ("num_workers", ctypes.c_int32),
        ("stream", ctypes.c_void_p),
        ("workspace", ctypes.c_void_p),
        ("workspace_bytes", ctypes.c_size_t),
        ("timing_start", ctypes.c_void_p),
        ("timing_stop", ctypes.c_void_p),
    ]


_lib: ctypes.CDLL | None = None


def load(path: str = LIBRARY) -> ctypes.CDLL:
    """Load libsl (once). The HIP runtime torch already loaded is reused."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise ImportError(f"{path} is missing: build it with `python -m paper_2504_15930_amd.build`")
    lib = ctypes.CDLL(path)
    P = ctypes.c_void_p
    D = ctypes.POINTER(Desc)
    lib.sl_decode_attn_workspace_size.argtypes = [D, ctypes.POINTER(ctypes.c_size_t)]
    lib.sl_decode_attn_num_workers.argtypes = [D, ctypes.c_int32, ctypes.POINTER(ctypes.c_int32)]
    lib.sl_decode_attn.argtypes = [D, P, P, P, P, P, ctypes.c_float, P]
    lib.sl_decode_attn_fp8.argtypes = [D, P, P, P, P, P, P, P, ctypes.c_float, P]
    lib.sl_kv_append.argtypes = [D, P, P, P, P, P, P]
    lib.sl_decode_attn_prefix.argtypes = [D, P, P, P, P, P, P, P, ctypes.c_int32, ctypes.c_float, P]
    lib.sl_decode_attn_prefix_fp8.argtypes = [D, P, P, P, P, P, P, P, P, P, ctypes.c_int32, ctypes.c_float, P]
    lib.sl_decode_attn_prefix_workspace_size.argtypes = [D, ctypes.c_int32, ctypes.POINTER(ctypes.c_size_t)]
    lib.sl_kv_append_fp8.argtypes = [D, P, P, P, P, P, P, P, P]
    lib.sl_decode_attn_noalloc.argtypes = [D, P, P, P, P, P, ctypes.c_float, P]
    lib.sl_decode_attn_fp4.argtypes = [D, P, P, P, P, ctypes.c_float, P]
    lib.sl_decode_attn_prefix_fp4.argtypes = [D, P, P, P, P, P, P, ctypes.c_int32, ctypes.c_float, P]
    lib.sl_kv_append_fp4.argtypes = [D, P, P, P, P, P]
    lib.sl_kv_write_fp4.argtypes = [D, P, P, P, ctypes.c_int32, P]
    lib.sl_kv_read_fp4.argtypes = [D, P, P, ctypes.c_int32, P, P]
    lib.sl_pages_extend.argtypes = [D, P, P, P, P, P, ctypes.c_int32, P, P, P, P]
    lib.sl_pages_release.argtypes = [D, P, P, P, P, P, P, P]
    lib.sl_status_string.argtypes = [ctypes.c_int32]
    lib.sl_status_string.restype = ctypes.c_char_p
    for name in EXPORTS[:-1]:
        getattr(lib, name).restype = ctypes.c_int
    _lib = lib
    return lib


def status_string(status: int) -> str:
    return load().sl_status_string(status).decode()


def make_desc(batch, num_q_heads, num_kv_heads, head_dim, page_size, max_blocks, num_pages,
              num_workers=0, stream=None, workspace=None, workspace_bytes=0,
              timing=None) -> Desc:
    d = Desc()
    d.batch, d.num_q_heads, d.num_kv_heads, d.head_dim = batch, num_q_heads, num_kv_heads, head_dim
    d.page_size, d.max_blocks_per_seq, d.num_pages = page_size, max_blocks, num_pages
    d.num_workers = num_workers
    d.stream = stream
    d.workspace = workspace
    d.workspace_bytes = workspace_bytes
    if timing is not None:
        d.timing_start, d.timing_stop = timing
    return d


def _check(status: int, where: str):
    if status != SL_OK:
        raise SlError(status, where)


def workspace_size(desc: Desc) -> int:
    n = ctypes.c_size_t(0)
    _check(load().sl_decode_attn_workspace_size(ctypes.byref(desc), ctypes.byref(n)),
           "sl_decode_attn_workspace_size")
    return n.value


def num_workers(desc: Desc, fp8: bool = False) -> int:
    n = ctypes.c_int32(0)
    _check(load().sl_decode_attn_num_workers(ctypes.byref(desc), int(fp8), ctypes.byref(n)),
           "sl_decode_attn_num_workers")
    return n.value


# Host time per call counts: a small step's kernels take less than the calls
# around them (18.1 us per call of 8 short sequences, 7.6 of them the library's
# two launches). A device context costs 1.4 us and a Stream object 1.9, so the
# one is entered only when the tensors' device is not the current one, and the
# stream is asked for as the raw handle (0.1 us); the workspace sizes of the
# shapes in use are kept.
_no_context = contextlib.nullcontext()


def _device(index: int):
    return _no_context if torch.cuda.current_device() == index else torch.cuda.device(index)


def _stream(index: int) -> int:
    """Raw handle of the current stream of GPU ``index``."""
    return torch._C._cuda_getCurrentRawStream(index)


@functools.lru_cache(maxsize=256)
def _workspace_bytes(index: int, *sizes) -> int:
    """``workspace_size`` for ``make_desc``'s sizes on GPU ``index`` (current): they decide it alone."""
    return workspace_size(make_desc(*sizes))


@functools.lru_cache(maxsize=256)
def _prefix_workspace_bytes(index: int, num_groups: int, *sizes) -> int:
    desc, need = make_desc(*sizes), ctypes.c_size_t(0)
    _check(load().sl_decode_attn_prefix_workspace_size(ctypes.byref(desc), num_groups, ctypes.byref(need)),
           "sl_decode_attn_prefix_workspace_size")
    return need.value


_workspaces: dict[tuple[int, int, int], torch.Tensor] = {}


def _workspace(index: int, stream: int, nbytes: int) -> torch.Tensor:
    """A cached scratch buffer of at least ``nbytes`` (256-byte aligned by torch) per (GPU,
    current stream, host thread). Calls of one thread on one stream run one after the other, so they
    may share a buffer; calls on two streams could overlap, and of two threads' calls on one stream
    the kernels could alternate (a call is a split and a merge). The buffer is allocated
    while its stream is current, so when it is replaced by a larger one torch's allocator hands
    its memory out again only in that stream's order, after the kernels that used it.

    A graph's replays are in no such order, and outlive the buffer that was cached when it was
    captured. So a call that is being captured gets a buffer of its own, out of the graph's memory
    pool: torch keeps that for as long as the graph, and shares it with no other graph unasked."""
    if torch.cuda.is_current_stream_capturing():
        return torch.empty(max(nbytes, 256), dtype=torch.uint8, device=torch.device("cuda", index))
    key = (index, stream, threading.get_ident())
    ws = _workspaces.get(key)
    if ws is None or ws.numel() < nbytes:
        if ws is None:   # a new stream or thread: those of ended threads go
            alive = {t.ident for t in threading.enumerate()} | {key[2]}
            for k in list(_workspaces):
                if k[2] not in alive:
                    _workspaces.pop(k, None)
        ws = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=torch.device("cuda", index))
        _workspaces[key] = ws
    return ws


def _need(t: torch.Tensor, name: str, dtype, ndim: int):
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.dim() != ndim:
        raise ValueError(f"{name} must have {ndim} dims, got shape {tuple(t.shape)}")
    if not t.is_cuda:
        raise ValueError(f"{name} must be on a GPU (libsl has no CPU path)")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def _run(fp8, q, k_pages, v_pages, k_scales, v_scales, block_table, seq_lens, scale, out,
         num_workers_, workspace, timing):
    kv_dtype = torch.uint8 if fp8 else torch.bfloat16
    _need(q, "q", torch.bfloat16, 3)
    _need(k_pages, "k_pages", kv_dtype, 4)
    _need(v_pages, "v_pages", kv_dtype, 4)
    _need(block_table, "block_table", torch.int32, 2)
    _need(seq_lens, "seq_lens", torch.int32, 1)
    if fp8:
        _need(k_scales, "k_scales", torch.float32, 2)
        _need(v_scales, "v_scales", torch.float32, 2)
    B, Hq, D = q.shape
    N, Hkv, P, D2 = k_pages.shape
    if D2 != D or tuple(v_pages.shape) != tuple(k_pages.shape):
        raise ValueError("q, k_pages and v_pages disagree on shape")
    if block_table.shape[0] != B or seq_lens.shape[0] != B:
        raise ValueError("block_table / seq_lens rows must equal the batch")
    if fp8 and (tuple(k_scales.shape) != (N, Hkv) or tuple(v_scales.shape) != (N, Hkv)):
        raise ValueError("scales must have shape [num_pages, num_kv_heads]")
    if out is None:
        out = torch.empty_like(q)
    else:
        _need(out, "out", torch.bfloat16, 3)
        if out.shape != q.shape:
            raise ValueError("out must have the shape of q")
    index = q.get_device()
    with _device(index):
        stream = _stream(index)
        sizes = (B, Hq, Hkv, D, P, block_table.shape[1], N, num_workers_)
        desc = make_desc(*sizes, stream)
        if B == 0:
            return out
        need = _workspace_bytes(index, *sizes)
        ws = workspace if workspace is not None else _workspace(index, stream, need)
        desc.workspace = ws.data_ptr()
        desc.workspace_bytes = ws.numel() * ws.element_size()
        if timing is not None:
            desc.timing_start, desc.timing_stop = timing
        lib = load()
        if fp8:
            st = lib.sl_decode_attn_fp8(ctypes.byref(desc), q.data_ptr(), k_pages.data_ptr(),
                                        v_pages.data_ptr(), k_scales.data_ptr(), v_scales.data_ptr(),
                                        block_table.data_ptr(), seq_lens.data_ptr(), float(scale),
                                        out.data_ptr())
            _check(st, "sl_decode_attn_fp8")
        else:
            st = lib.sl_decode_attn(ctypes.byref(desc), q.data_ptr(), k_pages.data_ptr(),
                                    v_pages.data_ptr(), block_table.data_ptr(), seq_lens.data_ptr(),
                                    float(scale), out.data_ptr())
            _check(st, "sl_decode_attn")
    return out


def decode_attn(q, k_pages, v_pages, block_table, seq_lens, scale, *, out=None, num_workers=0,
                workspace=None, timing=None) -> torch.Tensor:
    """``sl_decode_attn`` on torch tensors (bf16 KV cache); returns ``out`` [B, Hq, D] bf16.

    ``timing`` optionally holds two raw hipEvent handles recorded around the
    split-KV kernel. The call is asynchronous on the current stream.

    ``workspace`` (uint8 on the GPU) is the call's scratch; without it, the current stream's, or,
    captured by ``torch.cuda.graph``, memory of the graph's own pool. (A capture that was begun
    past torch has no such pool: such calls need a ``workspace``.)
    """
    return _run(False, q, k_pages, v_pages, None, None, block_table, seq_lens, scale, out,
                num_workers, workspace, timing)


def decode_attn_noalloc(q, k_pages, v_pages, block_table, seq_lens, scale, *, out=None,
                        num_workers=0) -> torch.Tensor:
    """``sl_decode_attn_noalloc``: ``sl_decode_attn`` with the library's fixed scratch array instead
    of a workspace (the call allocates nothing). Calls on one GPU must not overlap in time."""
    _need(q, "q", torch.bfloat16, 3)
    _need(k_pages, "k_pages", torch.bfloat16, 4)
    _need(v_pages, "v_pages", torch.bfloat16, 4)
    _need(block_table, "block_table", torch.int32, 2)
    _need(seq_lens, "seq_lens", torch.int32, 1)
    B, Hq, D = q.shape
    N, Hkv, P, D2 = k_pages.shape
    if D2 != D or tuple(v_pages.shape) != tuple(k_pages.shape):
        raise ValueError("q, k_pages and v_pages disagree on shape")
    if block_table.shape[0] != B or seq_lens.shape[0] != B:
        raise ValueError("block_table / seq_lens rows must equal the batch")
    if out is None:
        out = torch.empty_like(q)
    else:
        _need(out, "out", torch.bfloat16, 3)
        if out.shape != q.shape:
            raise ValueError("out must have the shape of q")
    index = q.get_device()
    with _device(index):
        desc = make_desc(B, Hq, Hkv, D, P, block_table.shape[1], N, num_workers, _stream(index))
        _check(load().sl_decode_attn_noalloc(ctypes.byref(desc), q.data_ptr(), k_pages.data_ptr(),
                                             v_pages.data_ptr(), block_table.data_ptr(), seq_lens.data_ptr(),
                                             float(scale), out.data_ptr()),
               "sl_decode_attn_noalloc")
    return out


def decode_attn_fp8(q, k_pages, v_pages, k_scales, v_scales, block_table, seq_lens, scale, *,
                    out=None, num_workers=0, workspace=None, timing=None) -> torch.Tensor:
    """``sl_decode_attn_fp8``: K/V pages are uint8 E4M3 codes with fp32 [N, Hkv] scales."""
    return _run(True, q, k_pages, v_pages, k_scales, v_scales, block_table, seq_lens, scale, out,
                num_workers, workspace, timing)


def run_batch(batch, **kw) -> torch.Tensor:
    """Decode attention on an ``inputs.Batch`` (dispatches on its KV dtype)."""
    if batch.kv_dtype == "e4m3":
        return decode_attn_fp8(batch.q, batch.k_pages, batch.v_pages, batch.k_scales,
                               batch.v_scales, batch.block_table, batch.seq_lens, batch.scale, **kw)
    return decode_attn(batch.q, batch.k_pages, batch.v_pages, batch.block_table, batch.seq_lens,
                       batch.scale, **kw)


def kv_append(k_new, v_new, block_table, seq_lens, k_pages, v_pages, *, k_scales=None,
              v_scales=None, num_q_heads=None, timing=None):
    """``sl_kv_append`` / ``sl_kv_append_fp8`` on torch tensors, in place.

    ``k_new``/``v_new``: bf16 [B, Hkv, D] rows of the step's new token;
    ``seq_lens`` already counts it. A uint8 page pool selects the E4M3 path,
    which needs fp32 ``k_scales``/``v_scales`` [N, Hkv] (updated in place).
    Asynchronous on the current stream.
    """
    fp8 = k_pages.dtype == torch.uint8
    kv_dtype = torch.uint8 if fp8 else torch.bfloat16
    _need(k_new, "k_new", torch.bfloat16, 3)
    _need(v_new, "v_new", torch.bfloat16, 3)
    _need(k_pages, "k_pages", kv_dtype, 4)
    _need(v_pages, "v_pages", kv_dtype, 4)
    _need(block_table, "block_table", torch.int32, 2)
    _need(seq_lens, "seq_lens", torch.int32, 1)
    if fp8:
        _need(k_scales, "k_scales", torch.float32, 2)
        _need(v_scales, "v_scales", torch.float32, 2)
    B, Hkv, D = k_new.shape
    N, Hkv2, P, D2 = k_pages.shape
    if (Hkv2, D2) != (Hkv, D) or tuple(v_new.shape) != (B, Hkv, D) or v_pages.shape != k_pages.shape:
        raise ValueError("k_new / v_new / pages disagree on shape")
    if block_table.shape[0] != B or seq_lens.shape[0] != B:
        raise ValueError("block_table / seq_lens rows must equal the batch")
    if fp8 and (tuple(k_scales.shape) != (N, Hkv) or tuple(v_scales.shape) != (N, Hkv)):
        raise ValueError("scales must have shape [num_pages, num_kv_heads]")
    index = k_new.get_device()
    with _device(index):
        desc = make_desc(B, num_q_heads or Hkv, Hkv, D, P, block_table.shape[1], N, 0, _stream(index))
        if timing is not None:
            desc.timing_start, desc.timing_stop = timing
        lib = load()
        if fp8:
            st = lib.sl_kv_append_fp8(ctypes.byref(desc), k_new.data_ptr(), v_new.data_ptr(),
                                      block_table.data_ptr(), seq_lens.data_ptr(), k_pages.data_ptr(),
                                      v_pages.data_ptr(), k_scales.data_ptr(), v_scales.data_ptr())
            _check(st, "sl_kv_append_fp8")
        else:
            st = lib.sl_kv_append(ctypes.byref(desc), k_new.data_ptr(), v_new.data_ptr(),
                                  block_table.data_ptr(), seq_lens.data_ptr(), k_pages.data_ptr(),
                                  v_pages.data_ptr())
            _check(st, "sl_kv_append")


def _run_prefix(fp8, q, k_pages, v_pages, k_scales, v_scales, block_table, seq_lens, scale, group_start,
                shared_pages, out, num_workers, workspace, timing):
    kv_dtype = torch.uint8 if fp8 else torch.bfloat16
    _need(q, "q", torch.bfloat16, 3)
    _need(k_pages, "k_pages", kv_dtype, 4)
    _need(v_pages, "v_pages", kv_dtype, 4)
    _need(block_table, "block_table", torch.int32, 2)
    _need(seq_lens, "seq_lens", torch.int32, 1)
    _need(group_start, "group_start", torch.int32, 1)
    _need(shared_pages, "shared_pages", torch.int32, 1)
    if fp8:
        _need(k_scales, "k_scales", torch.float32, 2)
        _need(v_scales, "v_scales", torch.float32, 2)
    ng = shared_pages.shape[0]
    if group_start.shape[0] != ng + 1:
        raise ValueError("group_start must have num_groups + 1 entries")
    B, Hq, D = q.shape
    N, Hkv, P, D2 = k_pages.shape
    if D2 != D or v_pages.shape != k_pages.shape or block_table.shape[0] != B or seq_lens.shape[0] != B:
        raise ValueError("shape mismatch")
    if fp8 and (tuple(k_scales.shape) != (N, Hkv) or tuple(v_scales.shape) != (N, Hkv)):
        raise ValueError("scales must have shape [num_pages, num_kv_heads]")
    if out is None:
        out = torch.empty_like(q)
    else:
        _need(out, "out", torch.bfloat16, 3)
        if out.shape != q.shape:
            raise ValueError("out must have the shape of q")
    lib = load()
    index = q.get_device()
    with _device(index):
        stream = _stream(index)
        sizes = (B, Hq, Hkv, D, P, block_table.shape[1], N, num_workers)
        desc = make_desc(*sizes, stream)
        if B == 0:
            return out
        need = _prefix_workspace_bytes(index, ng, *sizes)
        ws = workspace if workspace is not None else _workspace(index, stream, need)
        desc.workspace = ws.data_ptr()
        desc.workspace_bytes = ws.numel() * ws.element_size()
        if timing is not None:
            desc.timing_start, desc.timing_stop = timing
        if fp8:
            _check(lib.sl_decode_attn_prefix_fp8(ctypes.byref(desc), q.data_ptr(), k_pages.data_ptr(),
                                                 v_pages.data_ptr(), k_scales.data_ptr(), v_scales.data_ptr(),
                                                 block_table.data_ptr(), seq_lens.data_ptr(),
                                                 group_start.data_ptr(), shared_pages.data_ptr(), ng,
                                                 float(scale), out.data_ptr()),
                   "sl_decode_attn_prefix_fp8")
        else:
            _check(lib.sl_decode_attn_prefix(ctypes.byref(desc), q.data_ptr(), k_pages.data_ptr(),
                                             v_pages.data_ptr(), block_table.data_ptr(), seq_lens.data_ptr(),
                                             group_start.data_ptr(), shared_pages.data_ptr(), ng, float(scale),
                                             out.data_ptr()),
                   "sl_decode_attn_prefix")
    return out


def decode_attn_prefix(q, k_pages, v_pages, block_table, seq_lens, scale, group_start, shared_pages, *,
                       out=None, num_workers=0, workspace=None, timing=None) -> torch.Tensor:
    """``sl_decode_attn_prefix``: decode attention reading each group's shared pages once.

    ``group_start`` (int32 [G+1]) and ``shared_pages`` (int32 [G]) are device tensors;
    consecutive sequences of a group share their first ``shared_pages[k]`` pages.
    """
    return _run_prefix(False, q, k_pages, v_pages, None, None, block_table, seq_lens, scale, group_start,
                       shared_pages, out, num_workers, workspace, timing)


def decode_attn_prefix_fp8(q, k_pages, v_pages, k_scales, v_scales, block_table, seq_lens, scale, group_start,
                           shared_pages, *, out=None, num_workers=0, workspace=None, timing=None) -> torch.Tensor:
    """``sl_decode_attn_prefix_fp8``: prefix sharing over uint8 E4M3 pages with fp32 [N, Hkv] scales."""
    return _run_prefix(True, q, k_pages, v_pages, k_scales, v_scales, block_table, seq_lens, scale, group_start,
                       shared_pages, out, num_workers, workspace, timing)


# The 4-bit cache: one uint8 record of 17 D bytes per (page, KV head), as include/sl.h lays it out.

def fp4_record_bytes(head_dim: int) -> int:
    """Bytes of a page-head record of the 4-bit cache (16 tokens, keys and values)."""
    return 17 * head_dim


def _ptr(t: torch.Tensor, name: str, dtype, shape, index: int) -> int:
    """Address of ``t``, which must have this dtype and exact shape, contiguous, on GPU ``index``. (One pass over
    what decides it, 0.4 us; which of them failed is worked out only then.)"""
    try:
        if t.dtype is dtype and t.shape == shape and t.get_device() == index >= 0 and t.is_contiguous():
            return t.data_ptr()
    except AttributeError:
        pass
    _need(t, name, dtype, len(shape))
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    raise ValueError(f"{name} must be on cuda:{index} with the others, is on {t.device}")


def _refuse(*args):
    """Raise for whichever of the (tensor, name, dtype, dims) is not what it must be."""
    for a in args:
        _need(*a)
    raise ValueError("the arguments disagree on shape")


_BAD_SIZES = (AttributeError, IndexError, TypeError, ValueError)   # what asking a wrong argument for its sizes raises


# csrc/binding.cpp, bound to the library that ``load`` gives. Each of its functions makes one call of its kind on
# contiguous tensors of the current device, without timing events, and returns None, nothing done, for any other; the
# Python below then makes it, or says what is wrong with it. Time per call, 8 requests: attention 9.9 us by Python
# alone, 5.3 here; append 7.5 and 3.6, read 9.5 and 5.1, pages_extend 11.4 and 5.2, pages_release 10.2 and 4.9.
_fast = None


class _NoBinding:
    """In place of a binding that does not load: declines every call."""

    def __getattr__(self, name):
        return lambda *args: None


def _binding():
    global _fast
    if _fast is None:
        lib = load()
        try:
            from . import _binding as fast
        except ImportError as e:   # not built, or for another torch
            warnings.warn(f"calls of the 4-bit cache and the page bookkeeping take 4 to 6 us more: no _binding.so ({e}); "
                          "build it with `python -m paper_2504_15930_amd.build`", RuntimeWarning, stacklevel=3)
            _fast = _NoBinding()
            return _fast
        names = ("sl_decode_attn_fp4", "sl_decode_attn_prefix_fp4", "sl_decode_attn_workspace_size",
                 "sl_decode_attn_prefix_workspace_size", "sl_kv_append_fp4", "sl_kv_write_fp4", "sl_kv_read_fp4",
                 "sl_pages_extend", "sl_pages_release")
        fast.bind({n: ctypes.cast(getattr(lib, n), ctypes.c_void_p).value for n in names}, _workspaces, _workspace, _check)
        _fast = fast
    return _fast


def _run_fp4(q, kv_pages, block_table, seq_lens, scale, groups, out, num_workers, workspace, timing):
    try:
        (B, Hq, D), (N, Hkv, _), (_, blocks), index = q.shape, kv_pages.shape, block_table.shape, q.get_device()
        ng = 0 if groups is None else groups[1].shape[0]
    except _BAD_SIZES:
        _refuse((q, "q", torch.bfloat16, 3), (kv_pages, "kv_pages", torch.uint8, 3),
                (block_table, "block_table", torch.int32, 2),
                *(((groups[1], "shared_pages", torch.int32, 1),) if groups is not None else ()))
    args = [_ptr(q, "q", torch.bfloat16, (B, Hq, D), index),
            _ptr(kv_pages, "kv_pages", torch.uint8, (N, Hkv, 17 * D), index),
            _ptr(block_table, "block_table", torch.int32, (B, blocks), index),
            _ptr(seq_lens, "seq_lens", torch.int32, (B,), index)]
    sizes = (B, Hq, Hkv, D, PAGE_SIZE, blocks, N, num_workers)
    if groups is not None:
        args += [_ptr(groups[0], "group_start", torch.int32, (ng + 1,), index),
                 _ptr(groups[1], "shared_pages", torch.int32, (ng,), index), ng]
    if torch._C._cuda_getDevice() != index:
        with torch.cuda.device(index):
            return _run_fp4(q, kv_pages, block_table, seq_lens, scale, groups, out, num_workers, workspace, timing)
    if out is None:
        out = torch.empty_like(q)
        out_ptr = out.data_ptr()
    else:
        out_ptr = _ptr(out, "out", torch.bfloat16, (B, Hq, D), index)
    if B == 0:
        return out
    stream = _stream(index)
    if workspace is None:
        workspace = _workspace(index, stream, _workspace_bytes(index, *sizes) if groups is None else
                               _prefix_workspace_bytes(index, ng, *sizes))
    desc = Desc(*sizes, stream, workspace.data_ptr(), workspace.numel() * workspace.element_size(), *(timing or ()))
    name = "sl_decode_attn_fp4" if groups is None else "sl_decode_attn_prefix_fp4"
    _check(getattr(_lib or load(), name)(ctypes.byref(desc), *args, float(scale), out_ptr), name)
    return out


def decode_attn_fp4(q, kv_pages, block_table, seq_lens, scale, *, out=None, num_workers=0, workspace=None,
                    timing=None) -> torch.Tensor:
    """``sl_decode_attn_fp4``: decode attention over a 4-bit cache, ``kv_pages`` uint8
    [num_pages, Hkv, ``fp4_record_bytes(D)``]; otherwise as ``decode_attn``."""
    if workspace is None and timing is None:
        done = (_fast or _binding()).attn(q, kv_pages, block_table, seq_lens, scale, None, None, out, num_workers)
        if done is not None:
            return done
    return _run_fp4(q, kv_pages, block_table, seq_lens, scale, None, out, num_workers, workspace, timing)


def decode_attn_prefix_fp4(q, kv_pages, block_table, seq_lens, scale, group_start, shared_pages, *, out=None,
                           num_workers=0, workspace=None, timing=None) -> torch.Tensor:
    """``sl_decode_attn_prefix_fp4``: prefix sharing over a 4-bit cache; groups as ``decode_attn_prefix``."""
    if workspace is None and timing is None and shared_pages is not None:
        done = (_fast or _binding()).attn(q, kv_pages, block_table, seq_lens, scale, group_start, shared_pages, out,
                                          num_workers)
        if done is not None:
            return done
    return _run_fp4(q, kv_pages, block_table, seq_lens, scale, (group_start, shared_pages), out, num_workers,
                    workspace, timing)


def kv_append_fp4(k_new, v_new, block_table, seq_lens, kv_pages, *, timing=None):
    """``sl_kv_append_fp4``: a decode step's new rows [B, Hkv, D] (bf16) quantised into a 4-bit cache, in place;
    ``seq_lens`` already counts them. Asynchronous on the current stream."""
    if timing is None and (_fast or _binding()).append(k_new, v_new, block_table, seq_lens, kv_pages):
        return
    try:
        (B, Hkv, D), N, blocks, index = k_new.shape, kv_pages.shape[0], block_table.shape[1], k_new.get_device()
    except _BAD_SIZES:
        _refuse((k_new, "k_new", torch.bfloat16, 3), (kv_pages, "kv_pages", torch.uint8, 3),
                (block_table, "block_table", torch.int32, 2))
    args = (_ptr(k_new, "k_new", torch.bfloat16, (B, Hkv, D), index), _ptr(v_new, "v_new", torch.bfloat16, (B, Hkv, D), index),
            _ptr(block_table, "block_table", torch.int32, (B, blocks), index),
            _ptr(seq_lens, "seq_lens", torch.int32, (B,), index),
            _ptr(kv_pages, "kv_pages", torch.uint8, (N, Hkv, 17 * D), index))
    if torch._C._cuda_getDevice() != index:
        with torch.cuda.device(index):
            return kv_append_fp4(k_new, v_new, block_table, seq_lens, kv_pages, timing=timing)
    desc = Desc(B, Hkv, Hkv, D, PAGE_SIZE, blocks, N, 0, _stream(index), None, 0, *(timing or ()))
    _check((_lib or load()).sl_kv_append_fp4(ctypes.byref(desc), *args), "sl_kv_append_fp4")


def kv_write_fp4(k_new, v_new, slots, kv_pages, *, timing=None):
    """``sl_kv_write_fp4``: rows [T, Hkv, D] (bf16) quantised into the slots ``slots`` (int32 [T], page * 16 + slot in
    the page; negative: no token) of a 4-bit cache, in place. Asynchronous on the current stream."""
    if timing is None and (_fast or _binding()).write(k_new, v_new, slots, kv_pages):
        return
    try:
        (T, Hkv, D), N, index = k_new.shape, kv_pages.shape[0], k_new.get_device()
    except _BAD_SIZES:
        _refuse((k_new, "k_new", torch.bfloat16, 3), (kv_pages, "kv_pages", torch.uint8, 3))
    args = (_ptr(k_new, "k_new", torch.bfloat16, (T, Hkv, D), index), _ptr(v_new, "v_new", torch.bfloat16, (T, Hkv, D), index),
            _ptr(slots, "slots", torch.int32, (T,), index), T,
            _ptr(kv_pages, "kv_pages", torch.uint8, (N, Hkv, 17 * D), index))
    if torch._C._cuda_getDevice() != index:
        with torch.cuda.device(index):
            return kv_write_fp4(k_new, v_new, slots, kv_pages, timing=timing)
    desc = Desc(0, Hkv, Hkv, D, PAGE_SIZE, 1, N, 0, _stream(index), None, 0, *(timing or ()))
    _check((_lib or load()).sl_kv_write_fp4(ctypes.byref(desc), *args), "sl_kv_write_fp4")


def kv_read_fp4(slots, kv_pages, *, k_out=None, v_out=None, timing=None) -> tuple[torch.Tensor, torch.Tensor]:
    """``sl_kv_read_fp4``: the key and value rows (bf16 [T, Hkv, D]) in the slots ``slots`` (int32 [T]) of a 4-bit
    cache; zero rows for negative slots, NaN for slots past the pool. Asynchronous on the current stream."""
    if timing is None:
        done = (_fast or _binding()).read(slots, kv_pages, k_out, v_out)
        if done is not None:
            return done
    try:
        (N, Hkv, size), (T,), index = kv_pages.shape, slots.shape, kv_pages.get_device()
    except _BAD_SIZES:
        _refuse((kv_pages, "kv_pages", torch.uint8, 3), (slots, "slots", torch.int32, 1))
    D = size // 17
    pool = _ptr(kv_pages, "kv_pages", torch.uint8, (N, Hkv, 17 * D), index)
    at = _ptr(slots, "slots", torch.int32, (T,), index)
    if torch._C._cuda_getDevice() != index:
        with torch.cuda.device(index):
            return kv_read_fp4(slots, kv_pages, k_out=k_out, v_out=v_out, timing=timing)
    if k_out is None:
        k_out = torch.empty((T, Hkv, D), dtype=torch.bfloat16, device=kv_pages.device)
        k_ptr = k_out.data_ptr()
    else:
        k_ptr = _ptr(k_out, "k_out", torch.bfloat16, (T, Hkv, D), index)
    if v_out is None:
        v_out = torch.empty_like(k_out)
        v_ptr = v_out.data_ptr()
    else:
        v_ptr = _ptr(v_out, "v_out", torch.bfloat16, (T, Hkv, D), index)
    desc = Desc(0, Hkv, Hkv, D, PAGE_SIZE, 1, N, 0, _stream(index), None, 0, *(timing or ()))
    _check((_lib or load()).sl_kv_read_fp4(ctypes.byref(desc), pool, at, T, k_ptr, v_ptr), "sl_kv_read_fp4")
    return k_out, v_out


def pages_extend(seq_lens, new_tokens, block_table, free_pages, free_count, max_tokens, *, seq_lens_out=None,
                 free_count_out=None, token_start=None, slots=None):
    """``sl_pages_extend``: room for ``new_tokens`` [B] more tokens per request. Pages come from the top of the stack
    ``free_pages`` [num_pages] (the first ``free_count`` [1] of it are free) and are entered in ``block_table``, in
    place. Returns ``(seq_lens_out, token_start, slots, free_count_out)``: the new lengths [B], where each request's
    tokens begin in the slot map [B + 1], the slot map [max_tokens] (-1 past the last token), and the pages left.
    ``seq_lens_out`` and ``free_count_out`` may be the inputs themselves. All int32; asynchronous. (Four outputs made by
    the call lie in one allocation, which lasts as long as any of them: clone one that is kept when the slot map is not.)"""
    done = (_fast or _binding()).extend(seq_lens, new_tokens, block_table, free_pages, free_count, max_tokens,
                                        seq_lens_out, free_count_out, token_start, slots)
    if done is not None:
        return done
    try:
        (B,), blocks, (N,), index = seq_lens.shape, block_table.shape[1], free_pages.shape, seq_lens.get_device()
    except _BAD_SIZES:
        _refuse((seq_lens, "seq_lens", torch.int32, 1), (block_table, "block_table", torch.int32, 2),
                (free_pages, "free_pages", torch.int32, 1))
    args = (_ptr(seq_lens, "seq_lens", torch.int32, (B,), index), _ptr(new_tokens, "new_tokens", torch.int32, (B,), index),
            _ptr(block_table, "block_table", torch.int32, (B, blocks), index),
            _ptr(free_pages, "free_pages", torch.int32, (N,), index),
            _ptr(free_count, "free_count", torch.int32, (1,), index), max_tokens)
    if torch._C._cuda_getDevice() != index:
        with torch.cuda.device(index):
            return pages_extend(seq_lens, new_tokens, block_table, free_pages, free_count, max_tokens,
                                seq_lens_out=seq_lens_out, free_count_out=free_count_out, token_start=token_start,
                                slots=slots)
    if not 0 <= max_tokens < 1 << 31:
        raise ValueError(f"max_tokens must lie in [0, 2^31), got {max_tokens}")
    if seq_lens_out is None and free_count_out is None and token_start is None and slots is None:
        # one allocation for all four
        room = torch.empty(2 * B + 2 + max_tokens, dtype=torch.int32, device=seq_lens.device)
        at = room.data_ptr()
        args += (at, at + 4 * (2 * B + 1 + max_tokens), at + 4 * B, at + 4 * (2 * B + 1))
        seq_lens_out, token_start, slots, free_count_out = room.split((B, B + 1, max_tokens, 1))
    else:
        new = lambda t, n: torch.empty(n, dtype=torch.int32, device=seq_lens.device) if t is None else t
        seq_lens_out, free_count_out = new(seq_lens_out, B), new(free_count_out, 1)
        token_start, slots = new(token_start, B + 1), new(slots, max_tokens)
        args += (_ptr(seq_lens_out, "seq_lens_out", torch.int32, (B,), index),
                 _ptr(free_count_out, "free_count_out", torch.int32, (1,), index),
                 _ptr(token_start, "token_start", torch.int32, (B + 1,), index),
                 _ptr(slots, "slots", torch.int32, (max_tokens,), index))
    desc = Desc(B, 1, 1, 64, PAGE_SIZE, blocks, N, 0, _stream(index))
    _check((_lib or load()).sl_pages_extend(ctypes.byref(desc), *args), "sl_pages_extend")
    return seq_lens_out, token_start, slots, free_count_out


def pages_release(finished, seq_lens, block_table, free_pages, free_count, *, seq_lens_out=None, free_count_out=None):
    """``sl_pages_release``: the pages of requests with ``finished`` [B] not 0 go back on the stack, in place, and
    their lengths become 0. Returns ``(seq_lens_out, free_count_out)``, which may be the inputs themselves, or, made by
    the call, lie in one allocation. A page that several rows share would come back once for each: keep such pages out of
    the released rows."""
    done = (_fast or _binding()).release(finished, seq_lens, block_table, free_pages, free_count, seq_lens_out,
                                         free_count_out)
    if done is not None:
        return done
    try:
        (B,), blocks, (N,), index = seq_lens.shape, block_table.shape[1], free_pages.shape, seq_lens.get_device()
    except _BAD_SIZES:
        _refuse((seq_lens, "seq_lens", torch.int32, 1), (block_table, "block_table", torch.int32, 2),
                (free_pages, "free_pages", torch.int32, 1))
    args = (_ptr(finished, "finished", torch.int32, (B,), index), _ptr(seq_lens, "seq_lens", torch.int32, (B,), index),
            _ptr(block_table, "block_table", torch.int32, (B, blocks), index),
            _ptr(free_pages, "free_pages", torch.int32, (N,), index),
            _ptr(free_count, "free_count", torch.int32, (1,), index))
    if torch._C._cuda_getDevice() != index:
        with torch.cuda.device(index):
            return pages_release(finished, seq_lens, block_table, free_pages, free_count, seq_lens_out=seq_lens_out,
                                 free_count_out=free_count_out)
    if seq_lens_out is None:
        seq_lens_out = torch.empty_like(seq_lens)
    if free_count_out is None:
        free_count_out = torch.empty_like(free_count)
    args += (_ptr(seq_lens_out, "seq_lens_out", torch.int32, (B,), index),
             _ptr(free_count_out, "free_count_out", torch.int32, (1,), index))
    desc = Desc(B, 1, 1, 64, PAGE_SIZE, blocks, N, 0, _stream(index))
    _check((_lib or load()).sl_pages_release(ctypes.byref(desc), *args), "sl_pages_release")
    return seq_lens_out, free_count_out
