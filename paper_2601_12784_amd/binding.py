"""ctypes binding of libsf_decode_attn.so (argument marshalling only).

The names mirror the C entry points declared in include/sf_decode_attn.h.
Every step of the computation runs in the HIP library; PyTorch only supplies
device memory and the stream. If the library is missing this module raises:
there is no fallback path.
"""
from __future__ import annotations

import contextlib
import ctypes
import os
import re
import threading
import weakref

import numpy as np
import torch

PKG = os.path.dirname(os.path.abspath(__file__))
# SF_DECODE_ATTN_LIB selects another build of the same library (the
# sanitized CPU-test copy of build.py --sanitize); default: the in-tree one.
LIB_PATH = os.environ.get("SF_DECODE_ATTN_LIB") or os.path.join(PKG, "libsf_decode_attn.so")
HEADER = os.path.join(os.path.dirname(PKG), "include", "sf_decode_attn.h")
PAGE = 16
ITEM_INTS = 8

STATUS = {0: "SF_OK", 1: "SF_ERR_INVALID_ARG", 2: "SF_ERR_UNSUPPORTED", 3: "SF_ERR_CAPACITY",
          4: "SF_ERR_PLAN_MISMATCH", 5: "SF_ERR_HIP"}
UNSUPPORTED, CAPACITY = 2, 3


class SfError(RuntimeError):
    def __init__(self, where: str, status: int):
        self.status = int(status)
        super().__init__(f"{where}: {STATUS.get(self.status, self.status)} ({status_string(self.status)})")


class sf_attn_desc(ctypes.Structure):
    _fields_ = [("num_seqs", ctypes.c_int32), ("num_q_heads", ctypes.c_int32),
                ("num_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("block_table_stride", ctypes.c_int32),
                ("num_pages", ctypes.c_int32), ("softmax_scale", ctypes.c_float)]


class sf_plan_opts(ctypes.Structure):
    _fields_ = [("num_cus", ctypes.c_int32), ("chunk_pages", ctypes.c_int32),
                ("workers_per_cu", ctypes.c_int32), ("min_chunk_pages", ctypes.c_int32),
                ("xcd_parity_skew", ctypes.c_int32)]


class sf_plan_info(ctypes.Structure):
    _fields_ = [("num_workers", ctypes.c_int32), ("num_work", ctypes.c_int32),
                ("num_combine", ctypes.c_int32), ("num_partials", ctypes.c_int32),
                ("chunk_pages", ctypes.c_int32), ("workers_per_group", ctypes.c_int32),
                ("work_bytes", ctypes.c_uint64), ("workspace_bytes", ctypes.c_uint64),
                ("desc_key", ctypes.c_uint64)]


class sf_extend_info(ctypes.Structure):
    _fields_ = [("num_items", ctypes.c_int32), ("tokens_per_item", ctypes.c_int32),
                ("num_q_rows", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("work_bytes", ctypes.c_uint64), ("desc_key", ctypes.c_uint64)]


class sf_store_info(ctypes.Structure):
    _fields_ = [("num_rows", ctypes.c_int32), ("num_q_rows", ctypes.c_int32), ("work_bytes", ctypes.c_uint64),
                ("desc_key", ctypes.c_uint64)]


class sf_weights_info(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("num_items", "num_merge", "num_slots", "item_pages", "num_q_rows",
                                              "steps")] + \
               [(n, ctypes.c_uint64) for n in ("work_bytes", "workspace_bytes", "desc_key")]


class sf_evict_info(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("num_seqs", "num_moves", "sinks", "recent", "boundary", "hole_pages", "num_long",
                                              "reserved")] + \
               [(n, ctypes.c_uint64) for n in ("work_bytes", "workspace_bytes", "desc_key")]


class sf_shared_info(ctypes.Structure):
    _fields_ = [("num_workers", ctypes.c_int32), ("num_work", ctypes.c_int32), ("num_merge", ctypes.c_int32),
                ("num_rows", ctypes.c_int32), ("workers_per_group", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("work_bytes", ctypes.c_uint64), ("workspace_bytes", ctypes.c_uint64), ("desc_key", ctypes.c_uint64)]


class sf_rotary_desc(ctypes.Structure):
    _fields_ = [("head_dim", ctypes.c_int32), ("rotary_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32),
                ("magnitude", ctypes.c_float)]


class sf_rotary_scaling(ctypes.Structure):
    _fields_ = [("factor", ctypes.c_double), ("trained_length", ctypes.c_double), ("low_turns", ctypes.c_double),
                ("high_turns", ctypes.c_double)]


class sf_sample_desc(ctypes.Structure):
    _fields_ = [("num_rows", ctypes.c_int32), ("vocab", ctypes.c_int32), ("row_stride", ctypes.c_int64),
                ("dtype", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class sf_runner_extras(ctypes.Structure):
    _fields_ = [("k_new", ctypes.c_void_p), ("v_new", ctypes.c_void_p), ("new_pages_host", ctypes.c_void_p),
                ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p), ("attn_start", ctypes.c_void_p),
                ("attn_end", ctypes.c_void_p)]


class sf_runner_memory(ctypes.Structure):
    _fields_ = [("pinned", ctypes.c_void_p), ("pinned_bytes", ctypes.c_uint64), ("device", ctypes.c_void_p),
                ("device_bytes", ctypes.c_uint64), ("need_slot", ctypes.c_uint64), ("need_device", ctypes.c_uint64),
                ("slots", ctypes.c_int32), ("device_per_call", ctypes.c_int32)]


class sf_cost_model(ctypes.Structure):
    _fields_ = [("k1", ctypes.c_double), ("k2", ctypes.c_double), ("k3", ctypes.c_double),
                ("k4", ctypes.c_double), ("k5", ctypes.c_double), ("kv_budget", ctypes.c_double)]


class sf_instance_state(ctypes.Structure):
    _fields_ = [("version", ctypes.c_int32), ("num_running", ctypes.c_int32),
                ("num_waiting", ctypes.c_int32), ("reserved", ctypes.c_int32), ("kv_cache", ctypes.c_double)]


class sf_trajectory(ctypes.Structure):
    _fields_ = [("version", ctypes.c_int32), ("reserved", ctypes.c_int32), ("length", ctypes.c_double)]


_lib = None


def lib():
    """Loads the HIP library (raises if it was not built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing; build it with `python -m paper_2601_12784_amd.build`")
    L = ctypes.CDLL(LIB_PATH)
    P = ctypes.POINTER
    vp = ctypes.c_void_p
    L.sf_decode_attn_plan.argtypes = [P(sf_attn_desc), vp, P(sf_plan_opts), vp, ctypes.c_uint64,
                                      P(sf_plan_info)]
    L.sf_decode_attn.argtypes = [P(sf_attn_desc), P(sf_plan_info), vp, vp, vp, vp, vp, vp, vp, vp,
                                 vp, ctypes.c_uint64, vp]
    L.sf_decode_attn_combine.argtypes = [P(sf_attn_desc), P(sf_plan_info), vp, vp, ctypes.c_uint64,
                                         vp, vp, vp]
    L.sf_decode_attn_scratch.argtypes = [P(sf_attn_desc), P(sf_plan_info), vp, vp, vp, vp, vp, vp, vp, vp]
    L.sf_debug_gather_kv.argtypes = [P(sf_attn_desc), vp, vp, vp, ctypes.c_int32, ctypes.c_int32,
                                     ctypes.c_int32, vp, vp, vp]
    L.sf_decode_attn_append.argtypes = [P(sf_attn_desc), P(sf_plan_info), vp, vp, vp, vp, vp, vp, vp, vp,
                                        vp, vp, vp, vp, ctypes.c_uint64, vp]
    L.sf_runner_create.argtypes = [P(sf_attn_desc), P(sf_plan_opts), P(vp)]
    L.sf_runner_reserve.argtypes = [vp, ctypes.c_uint64, ctypes.c_uint64, ctypes.c_int32, vp]
    L.sf_runner_reserve_batch.argtypes = [vp, vp, ctypes.c_int32, vp]
    L.sf_runner_reserve.restype = ctypes.c_int
    L.sf_runner_destroy.argtypes = [vp]
    L.sf_runner_destroy.restype = None
    L.sf_runner_step.argtypes = [vp, P(sf_attn_desc), vp, vp, vp, vp, vp, vp, vp, P(sf_runner_extras), vp,
                                 P(sf_plan_info)]
    L.sf_debug_stream_read.argtypes = [vp, ctypes.c_uint64, vp, ctypes.c_int32, vp, vp, vp]
    L.sf_decode_attn_fp8.argtypes = [P(sf_attn_desc), P(sf_plan_info), vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp,
                                     ctypes.c_uint64, vp]
    L.sf_kv_quantize_fp8.argtypes = [P(sf_attn_desc), vp, vp, vp, vp, ctypes.c_int32, vp, vp, vp, vp, vp]
    L.sf_extend_attn_plan.argtypes = [P(sf_attn_desc), vp, vp, vp, ctypes.c_uint64, P(sf_extend_info)]
    L.sf_extend_attn.argtypes = [P(sf_attn_desc), P(sf_extend_info), vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp]
    L.sf_runner_extend.argtypes = [vp, P(sf_attn_desc), vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, P(sf_runner_memory),
                                   vp, P(sf_extend_info)]
    L.sf_debug_runner_reserve.argtypes = [P(sf_attn_desc), P(sf_plan_opts), ctypes.c_uint64, ctypes.c_uint64, ctypes.c_int32,
                                          ctypes.c_int64, vp]
    L.sf_debug_extend_plan.argtypes = [P(sf_attn_desc), vp, vp, ctypes.c_int32, ctypes.c_int32, vp, ctypes.c_uint64, vp]
    L.sf_runner_plan.argtypes = [P(sf_attn_desc), vp, P(sf_plan_opts), ctypes.c_int32, vp, ctypes.c_uint64,
                                 P(sf_plan_info)]
    L.sf_page_pool_create.argtypes = [ctypes.c_int32, P(vp)]
    L.sf_page_pool_destroy.argtypes = [vp]
    L.sf_page_pool_destroy.restype = None
    L.sf_page_pool_available.argtypes = [vp]
    L.sf_page_pool_available.restype = ctypes.c_int32
    for fn in ("sf_page_pool_claim", "sf_page_pool_release"):
        getattr(L, fn).argtypes = [vp, vp, ctypes.c_int32]
    L.sf_page_pool_alloc.argtypes = [vp, ctypes.c_int32, vp]
    L.sf_page_pool_share.argtypes = [vp, vp, ctypes.c_int32]
    i32, u64, desc = ctypes.c_int32, ctypes.c_uint64, P(sf_attn_desc)
    L.sf_kv_store_fp8_plan.argtypes = [desc, vp, vp, vp, u64, P(sf_store_info)]
    L.sf_kv_store_fp8.argtypes = [desc, P(sf_store_info)] + [vp] * 11
    L.sf_key_weights_plan.argtypes = [desc, vp, vp, vp, vp, P(sf_plan_opts), vp, u64, P(sf_weights_info)]
    L.sf_key_weights.argtypes = [desc, P(sf_weights_info)] + [vp] * 11 + [u64, vp]
    L.sf_kv_evict_plan.argtypes = [desc, vp, vp, vp, i32, i32, vp, u64, P(sf_evict_info)]
    L.sf_kv_evict.argtypes = [desc, P(sf_evict_info)] + [vp] * 12 + [u64, vp]
    L.sf_runner_store_fp8.argtypes = [vp, desc] + [vp] * 11
    L.sf_runner_key_weights.argtypes = [vp, desc] + [vp] * 13
    L.sf_runner_evict.argtypes = [vp, desc, vp, vp, vp, i32, i32] + [vp] * 10
    L.sf_extend_attn_fp8.argtypes = [desc, P(sf_extend_info)] + [vp] * 9 + [i32, vp, vp]
    L.sf_runner_extend_fp8.argtypes = [vp, desc] + [vp] * 10 + [P(sf_runner_memory), vp, P(sf_extend_info), vp, vp, i32]
    i64, rope = ctypes.c_int64, P(sf_rotary_desc)
    L.sf_shared_attn_plan.argtypes = [desc, vp, i32, vp, vp, i32, P(sf_plan_opts), vp, u64, P(sf_shared_info)]
    L.sf_shared_attn.argtypes = [desc, P(sf_shared_info)] + [vp] * 9 + [i32, vp, vp, u64, vp]
    L.sf_runner_shared.argtypes = [vp, desc, vp, i32] + [vp] * 9 + [i32, vp, vp]
    L.sf_rotary_frequencies.argtypes = [i32, ctypes.c_double, P(sf_rotary_scaling), vp]
    L.sf_rotary_turns.argtypes = [vp, i32, vp]
    L.sf_rotary.argtypes = [rope, i32, i32, i32, vp, vp] + [vp, i64] * 4 + [vp]
    L.sf_rotary_store_plan.argtypes = [desc, vp, vp, vp, vp, u64, P(sf_store_info)]
    L.sf_rotary_store.argtypes = [desc, rope, P(sf_store_info), vp, vp, vp] + [vp, i64] * 4 + [vp] * 5
    L.sf_runner_rotary_store.argtypes = [vp, desc, rope, vp, vp, vp, vp] + [vp, i64] * 4 + [vp] * 5
    L.sf_sample_workspace.argtypes = [P(sf_sample_desc), P(u64)]
    L.sf_sample.argtypes = [P(sf_sample_desc)] + [vp] * 10 + [u64, vp]
    L.sf_page_table_truncate.argtypes = [vp, vp, i32, i32, vp, vp]
    L.sf_page_table_step.argtypes = [vp, vp, ctypes.c_int32, ctypes.c_int32, vp, vp, ctypes.c_int32, vp]
    L.sf_cost_throughput.argtypes = [P(sf_cost_model), P(sf_instance_state)]
    L.sf_cost_marginal_gain.argtypes = [P(sf_cost_model), P(sf_instance_state), ctypes.c_double]
    L.sf_cost_ideal_gain.argtypes = [P(sf_cost_model), ctypes.c_double]
    for fn in ("sf_cost_throughput", "sf_cost_marginal_gain", "sf_cost_ideal_gain"):
        getattr(L, fn).restype = ctypes.c_double
    L.sf_check_block_table.argtypes = [P(sf_attn_desc), vp, vp, P(ctypes.c_int32)]
    L.sf_check_block_table.restype = ctypes.c_int
    L.sf_route.argtypes = [P(sf_cost_model), ctypes.c_double, ctypes.c_int32, vp, ctypes.c_int32, vp,
                           ctypes.c_int32, vp, P(ctypes.c_int32)]
    for fn in ("sf_decode_attn_plan", "sf_decode_attn", "sf_decode_attn_combine", "sf_debug_gather_kv",
               "sf_decode_attn_append", "sf_page_pool_create", "sf_page_pool_claim", "sf_page_pool_alloc",
               "sf_page_pool_release", "sf_page_table_step", "sf_route", "sf_extend_attn_plan",
               "sf_extend_attn", "sf_decode_attn_fp8", "sf_kv_quantize_fp8", "sf_runner_create",
               "sf_runner_step", "sf_runner_extend", "sf_runner_plan", "sf_debug_extend_plan",
               "sf_debug_runner_reserve", "sf_runner_reserve_batch", "sf_debug_stream_read", "sf_decode_attn_scratch",
               "sf_kv_store_fp8_plan", "sf_kv_store_fp8", "sf_key_weights_plan", "sf_key_weights", "sf_kv_evict_plan",
               "sf_kv_evict", "sf_runner_store_fp8", "sf_runner_key_weights", "sf_runner_evict",
               "sf_page_table_truncate", "sf_extend_attn_fp8", "sf_runner_extend_fp8", "sf_shared_attn_plan", "sf_shared_attn",
               "sf_runner_shared", "sf_rotary_frequencies", "sf_rotary_turns", "sf_rotary", "sf_rotary_store_plan",
               "sf_rotary_store", "sf_runner_rotary_store", "sf_sample_workspace", "sf_sample", "sf_page_pool_share"):
        getattr(L, fn).restype = ctypes.c_int
    L.sf_status_string.argtypes = [ctypes.c_int]
    L.sf_status_string.restype = ctypes.c_char_p
    L.sf_version.restype = ctypes.c_int32
    _lib = L
    return L


def header_functions() -> list[str]:
    """Names of the functions include/sf_decode_attn.h declares."""
    text = open(HEADER).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    return sorted(set(re.findall(r"\b(sf_[a-z0-9_]+)\s*\(", text)))


# SF_DEBUG_CHECKS=1: before each launch the classes below check every block-
# table entry the launch will read against the pool size (sf_check_block_table),
# on a host copy (DecodeLoopRunner keeps one; the others copy the device table
# back, which synchronizes: a debugging aid, not for timing).
DEBUG_CHECKS = os.environ.get("SF_DEBUG_CHECKS", "") not in ("", "0")


def check_block_table(desc: sf_attn_desc, block_table_host, seq_lens) -> None:
    """Raises SfError (naming the first bad sequence) unless every block-table
    entry a step over seq_lens reads lies in [0, desc.num_pages)."""
    bt = np.ascontiguousarray(block_table_host.cpu().numpy() if isinstance(block_table_host, torch.Tensor)
                              else block_table_host, dtype=np.int32)
    lens = np.ascontiguousarray(seq_lens, dtype=np.int32)
    if bt.shape != (desc.num_seqs, desc.block_table_stride) or lens.shape != (desc.num_seqs,):
        raise ValueError("block table or lengths do not match the descriptor")
    bad = ctypes.c_int32(-1)
    st = lib().sf_check_block_table(ctypes.byref(desc), bt.ctypes.data, lens.ctypes.data, ctypes.byref(bad))
    if st != 0:
        raise SfError(f"sf_check_block_table (sequence {bad.value})", st)


def _check_group_pages(desc, block_table, lens, offsets, shared) -> None:
    """check_block_table for a step of groups: of the shared pages, the first running member's entries count. An entry of
    another member there is not read; a page that is not the first member's is a mistake all the same."""
    bt = np.array(block_table.cpu().numpy() if isinstance(block_table, torch.Tensor) else block_table, dtype=np.int32)
    for i, tokens in enumerate(shared.tolist()):
        # (offsets out of order or range, members shorter than what they share: the call itself refuses them)
        a, b = (min(max(int(x), 0), lens.size) for x in offsets[i: i + 2])
        live, common = [s for s in range(a, b) if lens[s] > 0], max(tokens, 0) // PAGE
        for s in live[1:]:
            own, first = bt[s, :common], bt[live[0], :common]
            if np.any((own != first) & (own >= 0) & (own < desc.num_pages)):
                raise ValueError(f"sequence {s} does not start with the pages of sequence {live[0]}, of whose group it is")
            bt[s, :common] = first
    check_block_table(desc, bt, lens)


def _check_stored_pages(desc, block_table, lens, q_lens, new_pages) -> None:
    """check_block_table for a store: the entries of the new tokens' pages (the earlier ones are not read), less those that
    the call itself writes."""
    bt = np.array(block_table.cpu().numpy() if isinstance(block_table, torch.Tensor) else block_table, dtype=np.int32)
    named = np.zeros(lens.size, bool) if new_pages is None else new_pages >= 0
    first, end = np.maximum(lens - q_lens, 0) // PAGE, -(-lens.astype(np.int64) // PAGE) - named
    bt[np.arange(bt.shape[1])[None, :] < first[:, None]] = 0
    check_block_table(desc, bt, np.where((q_lens > 0) & (end > first), end * PAGE, 0))
    if new_pages is not None and np.any((new_pages < -1) | (new_pages >= desc.num_pages)):
        raise ValueError("new_pages holds a page id outside the pool")


def status_string(status: int) -> str:
    return lib().sf_status_string(int(status)).decode()


def version() -> int:
    return int(lib().sf_version())


def make_desc(num_seqs, num_q_heads, num_kv_heads, head_dim, block_table_stride, num_pages,
              softmax_scale, page_size=PAGE) -> sf_attn_desc:
    return sf_attn_desc(int(num_seqs), int(num_q_heads), int(num_kv_heads), int(head_dim),
                        int(page_size), int(block_table_stride), int(num_pages), float(softmax_scale))


def make_opts(num_cus=0, chunk_pages=0, workers_per_cu=0, min_chunk_pages=0, xcd_parity_skew=0):
    return sf_plan_opts(int(num_cus), int(chunk_pages), int(workers_per_cu), int(min_chunk_pages),
                        int(xcd_parity_skew))


def _addr(x) -> int | None:
    if x is None:
        return None
    if isinstance(x, torch.Tensor):
        return x.data_ptr()
    if isinstance(x, int):
        return x
    if isinstance(x, np.ndarray):
        return _host_addr(x)
    raise TypeError(type(x))


def _host_addr(a: np.ndarray) -> int:
    """a.ctypes.data without the object that a.ctypes makes (0.3 against 0.8 us)."""
    return a.__array_interface__["data"][0]


# The current stream's handle alone: torch.cuda.current_stream() takes 3 us to
# build its Stream object, a third of a short call's host time.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current_device = getattr(torch._C, "_cuda_getDevice", None)


def _current_stream(device=None) -> int:
    """Handle of the current stream of `device` (None, or without an index: the current device)."""
    if _raw_stream is None or _current_device is None or not torch.cuda.is_initialized():
        return torch.cuda.current_stream(device).cuda_stream
    index = None if device is None else device.index
    return _raw_stream(_current_device() if index is None else index)


_HERE = contextlib.nullcontext()


def _on_device(device):
    """torch.cuda.device(device), which costs 2 us, or nothing if that is the current one."""
    if _current_device is not None and torch.cuda.is_initialized() and _current_device() == device.index:
        return _HERE
    return torch.cuda.device(device)


def _made_on(stream, device):
    """Where a call on `stream` makes its tensors: memory of the current stream may still be in use there by what came before."""
    if stream is None:
        return _HERE
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(int(stream), device=device)
    return torch.cuda.stream(stream)


def _stream(stream) -> int | None:
    if stream is None:
        return _current_stream()
    if isinstance(stream, torch.cuda.Stream):
        return stream.cuda_stream
    return int(stream)


def _check(where, st):
    if st != 0:
        raise SfError(where, st)


def _dev(t: torch.Tensor, name: str, dtype, shape=None):
    if isinstance(t, torch.Tensor) and t.is_cuda and t.dtype is dtype and t.is_contiguous() and (shape is None or t.shape == shape):
        return t
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must live on the GPU (got {t.device})")
    if t.dtype is not dtype:
        raise ValueError(f"{name} must be {dtype} (got {t.dtype})")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")


# ----------------------------------------------------------------------------
# the C entry points
# ----------------------------------------------------------------------------
def sf_decode_attn_plan(desc: sf_attn_desc, seq_lens, opts: sf_plan_opts | None = None,
                        work_host=None):
    """Plans one decode step on the host. seq_lens: int32 host array/tensor.

    work_host: int32 host buffer (numpy or CPU tensor, pinned for async
    uploads) or None to allocate a numpy buffer of the right size.
    Returns (info, work_host)."""
    if isinstance(seq_lens, torch.Tensor):
        seq_lens = seq_lens.cpu().numpy()
    lens = np.ascontiguousarray(seq_lens, dtype=np.int32)
    if lens.shape != (desc.num_seqs,):
        raise ValueError("seq_lens must have num_seqs entries")
    info = sf_plan_info()
    L = lib()
    op = ctypes.byref(opts) if opts is not None else None
    if work_host is None:
        _check("sf_decode_attn_plan", L.sf_decode_attn_plan(ctypes.byref(desc), lens.ctypes.data, op,
                                                            None, 0, ctypes.byref(info)))
        work_host = np.empty(max(1, info.work_bytes // 4), dtype=np.int32)
    cap = work_host.numel() * 4 if isinstance(work_host, torch.Tensor) else work_host.nbytes
    _check("sf_decode_attn_plan", L.sf_decode_attn_plan(ctypes.byref(desc), lens.ctypes.data, op,
                                                        _addr(work_host), cap, ctypes.byref(info)))
    return info, work_host


def sf_decode_attn(desc, info, work_host, work_dev, q, k_pool, v_pool, block_table, out, lse=None,
                   workspace=None, stream=None):
    """Enqueues the attention kernel (and the work-list upload if work_host is given)."""
    b, hq, hkv, d = desc.num_seqs, desc.num_q_heads, desc.num_kv_heads, desc.head_dim
    _dev(q, "q", torch.bfloat16, (b, hq, d))
    _dev(k_pool, "k_pool", torch.bfloat16, (desc.num_pages, hkv, d // 8, PAGE, 8))
    _dev(v_pool, "v_pool", torch.bfloat16, (desc.num_pages, hkv, d, PAGE))
    _dev(block_table, "block_table", torch.int32, (b, desc.block_table_stride))
    _dev(out, "out", torch.float32, (b, hq, d))
    _dev(work_dev, "work_dev", torch.int32)
    if work_dev.numel() * 4 < info.work_bytes:
        raise ValueError("work_dev is smaller than the plan")
    if lse is not None:
        _dev(lse, "lse", torch.float32, (b, hq))
    ws_bytes = 0
    if workspace is not None:
        _dev(workspace, "workspace", workspace.dtype)
        ws_bytes = workspace.numel() * workspace.element_size()
    _check("sf_decode_attn", lib().sf_decode_attn(
        ctypes.byref(desc), ctypes.byref(info), _addr(work_host), _addr(work_dev), _addr(q),
        _addr(k_pool), _addr(v_pool), _addr(block_table), _addr(out), _addr(lse),
        _addr(workspace), ws_bytes, _stream(stream)))


def sf_decode_attn_fp8(desc, info, work_host, work_dev, q, k_pool8, v_pool8, k_scale, v_scale, block_table, out,
                       lse=None, workspace=None, stream=None):
    """Enqueues the attention kernel over an fp8 cache (uint8 pools, fp32 scales [N, Hkv])."""
    b, hq, hkv, d = desc.num_seqs, desc.num_q_heads, desc.num_kv_heads, desc.head_dim
    _dev(q, "q", torch.bfloat16, (b, hq, d))
    _dev(k_pool8, "k_pool8", torch.uint8, (desc.num_pages, hkv, PAGE * d))
    _dev(v_pool8, "v_pool8", torch.uint8, (desc.num_pages, hkv, PAGE * d))
    _dev(k_scale, "k_scale", torch.float32, (desc.num_pages, hkv))
    _dev(v_scale, "v_scale", torch.float32, (desc.num_pages, hkv))
    _dev(block_table, "block_table", torch.int32, (b, desc.block_table_stride))
    _dev(out, "out", torch.float32, (b, hq, d))
    _dev(work_dev, "work_dev", torch.int32)
    if work_dev.numel() * 4 < info.work_bytes:
        raise ValueError("work_dev is smaller than the plan")
    if lse is not None:
        _dev(lse, "lse", torch.float32, (b, hq))
    ws_bytes = 0
    if workspace is not None:
        _dev(workspace, "workspace", workspace.dtype)
        ws_bytes = workspace.numel() * workspace.element_size()
    _check("sf_decode_attn_fp8", lib().sf_decode_attn_fp8(
        ctypes.byref(desc), ctypes.byref(info), _addr(work_host), _addr(work_dev), _addr(q), _addr(k_pool8),
        _addr(v_pool8), _addr(k_scale), _addr(v_scale), _addr(block_table), _addr(out), _addr(lse),
        _addr(workspace), ws_bytes, _stream(stream)))


def sf_kv_quantize_fp8(desc, k_pool, v_pool, pages, valid_slots, k_pool8, v_pool8, k_scale, v_scale, stream=None):
    """Quantizes the listed pages (device int32 pages / valid_slots) of bf16 pools into fp8 ones."""
    hkv, d = desc.num_kv_heads, desc.head_dim
    _dev(k_pool, "k_pool", torch.bfloat16, (desc.num_pages, hkv, d // 8, PAGE, 8))
    _dev(v_pool, "v_pool", torch.bfloat16, (desc.num_pages, hkv, d, PAGE))
    _dev(pages, "pages", torch.int32)
    _dev(valid_slots, "valid_slots", torch.int32, tuple(pages.shape))
    _dev(k_pool8, "k_pool8", torch.uint8, (desc.num_pages, hkv, PAGE * d))
    _dev(v_pool8, "v_pool8", torch.uint8, (desc.num_pages, hkv, PAGE * d))
    _dev(k_scale, "k_scale", torch.float32, (desc.num_pages, hkv))
    _dev(v_scale, "v_scale", torch.float32, (desc.num_pages, hkv))
    _check("sf_kv_quantize_fp8", lib().sf_kv_quantize_fp8(
        ctypes.byref(desc), _addr(k_pool), _addr(v_pool), _addr(pages), _addr(valid_slots), int(pages.numel()),
        _addr(k_pool8), _addr(v_pool8), _addr(k_scale), _addr(v_scale), _stream(stream)))


def sf_decode_attn_append(desc, info, work_host, work_dev, q, k_new, v_new, new_pages, k_pool, v_pool,
                          block_table, out, lse, workspace=None, stream=None):
    """Enqueues an appending decode pass: attention over every sequence
    including its newest token (k_new, v_new: bf16 [B, Hkv, D]), then the
    merge of split sequences and the token stores into the pools and the
    block table (so no separate combine call). new_pages: device int32 [B]
    (-1 = no new page) or None."""
    b, hq, hkv, d = desc.num_seqs, desc.num_q_heads, desc.num_kv_heads, desc.head_dim
    _dev(q, "q", torch.bfloat16, (b, hq, d))
    _dev(k_new, "k_new", torch.bfloat16, (b, hkv, d))
    _dev(v_new, "v_new", torch.bfloat16, (b, hkv, d))
    if new_pages is not None:
        _dev(new_pages, "new_pages", torch.int32, (b,))
    _dev(k_pool, "k_pool", torch.bfloat16, (desc.num_pages, hkv, d // 8, PAGE, 8))
    _dev(v_pool, "v_pool", torch.bfloat16, (desc.num_pages, hkv, d, PAGE))
    _dev(block_table, "block_table", torch.int32, (b, desc.block_table_stride))
    _dev(out, "out", torch.float32, (b, hq, d))
    _dev(work_dev, "work_dev", torch.int32)
    if work_dev.numel() * 4 < info.work_bytes:
        raise ValueError("work_dev is smaller than the plan")
    if lse is None:
        raise ValueError("sf_decode_attn_append needs an lse buffer (the merge reads it back)")
    _dev(lse, "lse", torch.float32, (b, hq))
    ws_bytes = 0
    if workspace is not None:
        _dev(workspace, "workspace", workspace.dtype)
        ws_bytes = workspace.numel() * workspace.element_size()
    _check("sf_decode_attn_append", lib().sf_decode_attn_append(
        ctypes.byref(desc), ctypes.byref(info), _addr(work_host), _addr(work_dev), _addr(q), _addr(k_new),
        _addr(v_new), _addr(new_pages), _addr(k_pool), _addr(v_pool), _addr(block_table), _addr(out),
        _addr(lse), _addr(workspace), ws_bytes, _stream(stream)))


def _host_i32(x, name, n):
    """x as a host int32 array with an entry per sequence (None stays None)."""
    if x is None:
        return None
    if isinstance(x, torch.Tensor):
        x = x.cpu().numpy()
    x = x if isinstance(x, np.ndarray) and x.dtype == np.int32 and x.flags.c_contiguous else np.ascontiguousarray(x, np.int32)
    if x.shape != (n,):
        raise ValueError(f"{name} must have one entry per sequence")
    return x


def _planned(name, info, call, work_host):
    """call(work, capacity) into work_host, or into an array of the size it asks for."""
    if work_host is None:
        _check(name, call(None, 0))
        work_host = np.empty(max(1, info.work_bytes // 4), dtype=np.int32)
    cap = work_host.numel() * 4 if isinstance(work_host, torch.Tensor) else work_host.nbytes
    _check(name, call(_addr(work_host), cap))
    return info, work_host


def _check_work(info, work_dev, workspace=None):
    """The device work list and workspace of a planned call; returns the workspace's bytes."""
    _dev(work_dev, "work_dev", torch.int32)
    if work_dev.numel() * 4 < info.work_bytes:
        raise ValueError("work_dev is smaller than the plan")
    if workspace is None:
        return 0
    _dev(workspace, "workspace", workspace.dtype)
    return workspace.numel() * workspace.element_size()


def _check_pools(n, hkv, d, k_pool, v_pool, block_table, batch, fp8):
    """A cache's pools (v_pool may be None) and block table; fp8: (k_scale, v_scale), None for a bf16 cache."""
    if fp8 is None:
        _dev(k_pool, "k_pool", torch.bfloat16, (n, hkv, d // 8, PAGE, 8))
        if v_pool is not None:
            _dev(v_pool, "v_pool", torch.bfloat16, (n, hkv, d, PAGE))
    else:
        _dev(k_pool, "k_pool8", torch.uint8, (n, hkv, PAGE * d))
        _dev(fp8[0], "k_scale", torch.float32, (n, hkv))
        if v_pool is not None:
            _dev(v_pool, "v_pool8", torch.uint8, (n, hkv, PAGE * d))
            _dev(fp8[1], "v_scale", torch.float32, (n, hkv))
    _dev(block_table, "block_table", torch.int32, (batch, block_table.shape[1]))


def _check_slots(n, hkv, weights, weights_out, positions, positions_out=None):
    for t, name in ((weights, "weights"), (weights_out, "weights_out")):
        _dev(t, name, torch.float32, (n, hkv, PAGE))
    for t, name in ((positions, "positions"), (positions_out, "positions_out")):
        if t is not None:
            _dev(t, name, torch.int32, (n, hkv, PAGE))


def sf_kv_store_fp8_plan(desc, seq_lens, q_lens, work_host=None):
    """Plans the store of the last q_lens[s] of seq_lens[s] tokens into an fp8 cache. Returns (info, work_host)."""
    lens, qls = _host_i32(seq_lens, "seq_lens", desc.num_seqs), _host_i32(q_lens, "q_lens", desc.num_seqs)
    info = sf_store_info()
    return _planned("sf_kv_store_fp8_plan", info, lambda w, cap: lib().sf_kv_store_fp8_plan(
        ctypes.byref(desc), _host_addr(lens), _host_addr(qls), w, cap, ctypes.byref(info)), work_host)


def sf_kv_store_fp8(desc, info, work_host, work_dev, k_new, v_new, new_pages, k_pool8, v_pool8, k_scale, v_scale,
                    block_table, stream=None):
    """Enqueues the store of new tokens (k_new, v_new: bf16 [T, Hkv, D]) into an fp8 cache whose tiles' scales grow.
    new_pages: device int32 [B] (-1 = no new page) or None."""
    hkv, d = desc.num_kv_heads, desc.head_dim
    _dev(k_new, "k_new", torch.bfloat16, (info.num_q_rows, hkv, d))
    _dev(v_new, "v_new", torch.bfloat16, (info.num_q_rows, hkv, d))
    if new_pages is not None:
        _dev(new_pages, "new_pages", torch.int32, (desc.num_seqs,))
    _check_pools(desc.num_pages, hkv, d, k_pool8, v_pool8, block_table, desc.num_seqs, (k_scale, v_scale))
    _check_work(info, work_dev)
    _check("sf_kv_store_fp8", lib().sf_kv_store_fp8(
        ctypes.byref(desc), ctypes.byref(info), _addr(work_host), _addr(work_dev), _addr(k_new), _addr(v_new),
        _addr(new_pages), _addr(k_pool8), _addr(v_pool8), _addr(k_scale), _addr(v_scale), _addr(block_table),
        _stream(stream)))


def sf_key_weights_plan(desc, seq_lens, q_lens, held_lens=None, first_pos=None, opts=None, work_host=None):
    """Plans the weights pass of the last q_lens[s] of seq_lens[s] tokens' query rows. Returns (info, work_host)."""
    n = desc.num_seqs
    lens, qls = _host_i32(seq_lens, "seq_lens", n), _host_i32(q_lens, "q_lens", n)
    held, pos = _host_i32(held_lens, "held_lens", n), _host_i32(first_pos, "first_pos", n)
    info = sf_weights_info()
    return _planned("sf_key_weights_plan", info, lambda w, cap: lib().sf_key_weights_plan(
        ctypes.byref(desc), _host_addr(lens), _host_addr(qls), _addr(held), _addr(pos),
        None if opts is None else ctypes.byref(opts), w, cap, ctypes.byref(info)), work_host)


def sf_key_weights(desc, info, work_host, work_dev, q, lse, k_pool, block_table, weights, weights_out=None,
                   positions=None, k_scale=None, workspace=None, stream=None):
    """Enqueues the weights pass: every cached key's attention weight, summed over the rows of q (bf16 [T, Hq, D], lse
    fp32 [T, Hq]), added to `weights` (fp32 [N, Hkv, 16]) into weights_out (default: weights itself). positions
    (int32 [N, Hkv, 16]) takes those of keys weighed first. k_scale: k_pool is an fp8 cache's."""
    weights_out = weights if weights_out is None else weights_out
    hq, hkv, d = desc.num_q_heads, desc.num_kv_heads, desc.head_dim
    _dev(q, "q", torch.bfloat16, (info.num_q_rows, hq, d))
    _dev(lse, "lse", torch.float32, (info.num_q_rows, hq))
    _check_pools(desc.num_pages, hkv, d, k_pool, None, block_table, desc.num_seqs, None if k_scale is None else (k_scale,))
    _check_slots(desc.num_pages, hkv, weights, weights_out, positions)
    ws_bytes = _check_work(info, work_dev, workspace)
    _check("sf_key_weights", lib().sf_key_weights(
        ctypes.byref(desc), ctypes.byref(info), _addr(work_host), _addr(work_dev), _addr(q), _addr(lse), _addr(k_pool),
        _addr(k_scale), _addr(block_table), _addr(weights), _addr(weights_out), _addr(positions), _addr(workspace),
        ws_bytes, _stream(stream)))


def sf_kv_evict_plan(desc, seq_lens, keep_lens, ends=None, sinks=0, recent=0, work_host=None):
    """Plans an eviction from seq_lens[s] to at most keep_lens[s] tokens. Returns (info, work_host)."""
    n = desc.num_seqs
    lens, keep = _host_i32(seq_lens, "seq_lens", n), _host_i32(keep_lens, "keep_lens", n)
    end = _host_i32(ends, "ends", n)
    info = sf_evict_info()
    return _planned("sf_kv_evict_plan", info, lambda w, cap: lib().sf_kv_evict_plan(
        ctypes.byref(desc), _host_addr(lens), _host_addr(keep), _addr(end), int(sinks), int(recent), w, cap,
        ctypes.byref(info)), work_host)


def sf_kv_evict(desc, info, work_host, work_dev, k_pool, v_pool, block_table, weights, positions, weights_out=None,
                positions_out=None, fp8=None, workspace=None, stream=None):
    """Enqueues the eviction: every (sequence, KV head) keeps its heaviest tokens, in its first slots. fp8: (k_scale,
    v_scale) of an fp8 cache. weights_out and positions_out default to weights and positions themselves."""
    weights_out = weights if weights_out is None else weights_out
    positions_out = positions if positions_out is None else positions_out
    hkv, d = desc.num_kv_heads, desc.head_dim
    _check_pools(desc.num_pages, hkv, d, k_pool, v_pool, block_table, desc.num_seqs, fp8)
    _check_slots(desc.num_pages, hkv, weights, weights_out, positions, positions_out)
    ws_bytes = _check_work(info, work_dev, workspace)
    k_scale, v_scale = fp8 if fp8 is not None else (None, None)
    _check("sf_kv_evict", lib().sf_kv_evict(
        ctypes.byref(desc), ctypes.byref(info), _addr(work_host), _addr(work_dev), _addr(k_pool), _addr(v_pool),
        _addr(k_scale), _addr(v_scale), _addr(block_table), _addr(weights), _addr(positions), _addr(weights_out),
        _addr(positions_out), _addr(workspace), ws_bytes, _stream(stream)))


def sf_extend_attn_plan(desc: sf_attn_desc, seq_lens, q_lens, work_host=None):
    """Plans extend attention on the host. seq_lens (L_s, new tokens
    included) and q_lens (E_s): int32 host arrays. Returns (info, work_host)."""
    lens = np.ascontiguousarray(np.asarray(seq_lens), dtype=np.int32)
    qls = np.ascontiguousarray(np.asarray(q_lens), dtype=np.int32)
    if lens.shape != (desc.num_seqs,) or qls.shape != (desc.num_seqs,):
        raise ValueError("seq_lens and q_lens must have num_seqs entries")
    info = sf_extend_info()
    L = lib()
    if work_host is None:
        _check("sf_extend_attn_plan", L.sf_extend_attn_plan(ctypes.byref(desc), lens.ctypes.data, qls.ctypes.data,
                                                            None, 0, ctypes.byref(info)))
        work_host = np.empty(max(1, info.work_bytes // 4), dtype=np.int32)
    cap = work_host.numel() * 4 if isinstance(work_host, torch.Tensor) else work_host.nbytes
    _check("sf_extend_attn_plan", L.sf_extend_attn_plan(ctypes.byref(desc), lens.ctypes.data, qls.ctypes.data,
                                                        _addr(work_host), cap, ctypes.byref(info)))
    return info, work_host


def _check_extend(desc, rows, q, k_pool, v_pool, block_table, out, lse, k_new, v_new, fp8=None):
    """The tensors of an extend call over `rows` new tokens."""
    hq, hkv, d = desc.num_q_heads, desc.num_kv_heads, desc.head_dim
    _dev(q, "q", torch.bfloat16, (rows, hq, d))
    if fp8 is None:
        _dev(k_pool, "k_pool", torch.bfloat16, (desc.num_pages, hkv, d // 8, PAGE, 8))
        _dev(v_pool, "v_pool", torch.bfloat16, (desc.num_pages, hkv, d, PAGE))
    else:
        _check_pools(desc.num_pages, hkv, d, k_pool, v_pool, block_table, desc.num_seqs, fp8)
    _dev(block_table, "block_table", torch.int32, (desc.num_seqs, desc.block_table_stride))
    _dev(out, "out", out.dtype if fp8 is not None and out.dtype is torch.bfloat16 else torch.float32, (rows, hq, d))
    if lse is not None:
        _dev(lse, "lse", torch.float32, (rows, hq))
    if (k_new is None) != (v_new is None):
        raise ValueError("give both k_new and v_new, or neither")
    if k_new is not None:
        _dev(k_new, "k_new", torch.bfloat16, (rows, hkv, d))
        _dev(v_new, "v_new", torch.bfloat16, (rows, hkv, d))


def sf_extend_attn(desc, info, work_host, work_dev, q, k_pool, v_pool, block_table, out, lse=None,
                   k_new=None, v_new=None, stream=None):
    """Enqueues extend attention (after the store of k_new / v_new into the
    pools when both are given). q, out: [T, Hq, D]; k_new, v_new: [T, Hkv, D]."""
    _check_extend(desc, info.num_q_rows, q, k_pool, v_pool, block_table, out, lse, k_new, v_new)
    _dev(work_dev, "work_dev", torch.int32)
    if work_dev.numel() * 4 < info.work_bytes:
        raise ValueError("work_dev is smaller than the plan")
    _check("sf_extend_attn", lib().sf_extend_attn(
        ctypes.byref(desc), ctypes.byref(info), _addr(work_host), _addr(work_dev), _addr(q), _addr(k_new),
        _addr(v_new), _addr(k_pool), _addr(v_pool), _addr(block_table), _addr(out), _addr(lse),
        _stream(stream)))


def sf_extend_attn_fp8(desc, info, work_host, work_dev, q, k_pool8, v_pool8, k_scale, v_scale, block_table, out,
                       lse=None, stream=None):
    """Enqueues extend attention over an fp8 cache that holds the new tokens already (sf_kv_store_fp8). q, out:
    [T, Hq, D]; out fp32 or bf16."""
    _check_extend(desc, info.num_q_rows, q, k_pool8, v_pool8, block_table, out, lse, None, None, (k_scale, v_scale))
    _check_work(info, work_dev)
    _check("sf_extend_attn_fp8", lib().sf_extend_attn_fp8(
        ctypes.byref(desc), ctypes.byref(info), _addr(work_host), _addr(work_dev), _addr(q), _addr(k_pool8),
        _addr(v_pool8), _addr(k_scale), _addr(v_scale), _addr(block_table), _addr(out),
        int(out.dtype is torch.bfloat16), _addr(lse), _stream(stream)))


def sf_shared_attn_plan(desc, seq_lens, group_offsets, shared_lens, opts=None, work_host=None, fp8=False):
    """Plans a decode step of groups that share their first tokens: sequences group_offsets[i] .. group_offsets[i+1] - 1
    have shared_lens[i] of them in common. Returns (info, work_host)."""
    lens, offsets, shared = _host_groups(desc.num_seqs, seq_lens, group_offsets, shared_lens)
    info = sf_shared_info()
    return _planned("sf_shared_attn_plan", info, lambda w, cap: lib().sf_shared_attn_plan(
        ctypes.byref(desc), _host_addr(lens), shared.size, _host_addr(offsets), _host_addr(shared), int(fp8),
        None if opts is None else ctypes.byref(opts), w, cap, ctypes.byref(info)), work_host)


def _host_groups(n, seq_lens, group_offsets, shared_lens):
    lens = _host_i32(seq_lens, "seq_lens", n)
    shared = np.ascontiguousarray(shared_lens, dtype=np.int32)
    if shared.ndim != 1:
        raise ValueError("shared_lens must have one entry per group")
    return lens, _host_i32(group_offsets, "group_offsets", shared.size + 1), shared


def _check_step(desc, q, k_pool, v_pool, block_table, out, lse, fp8):
    b, hq, d = desc.num_seqs, desc.num_q_heads, desc.head_dim
    _dev(q, "q", torch.bfloat16, (b, hq, d))
    _dev(out, "out", torch.bfloat16 if out.dtype is torch.bfloat16 else torch.float32, (b, hq, d))
    if lse is not None:
        _dev(lse, "lse", torch.float32, (b, hq))
    _check_pools(desc.num_pages, desc.num_kv_heads, d, k_pool, v_pool, block_table, b, fp8)


def sf_shared_attn(desc, info, work_host, work_dev, q, k_pool, v_pool, block_table, out, lse=None, fp8=None,
                   workspace=None, stream=None):
    """Enqueues a decode step of groups that share their first tokens. out: fp32 or bf16 [B, Hq, D]; fp8: (k_scale,
    v_scale) of an fp8 cache."""
    _check_step(desc, q, k_pool, v_pool, block_table, out, lse, fp8)
    ws_bytes = _check_work(info, work_dev, workspace)
    k_scale, v_scale = fp8 if fp8 is not None else (None, None)
    _check("sf_shared_attn", lib().sf_shared_attn(
        ctypes.byref(desc), ctypes.byref(info), _addr(work_host), _addr(work_dev), _addr(q), _addr(k_pool), _addr(v_pool),
        _addr(k_scale), _addr(v_scale), _addr(block_table), _addr(out), int(out.dtype is torch.bfloat16), _addr(lse),
        _addr(workspace), ws_bytes, _stream(stream)))


def sf_rotary_frequencies(rotary_dim, base, scaling=None) -> np.ndarray:
    """The rotation's frequencies, radians per position (float64 [rotary_dim / 2]). scaling: a sf_rotary_scaling."""
    freq = np.empty(max(0, int(rotary_dim)) // 2, dtype=np.float64)
    _check("sf_rotary_frequencies", lib().sf_rotary_frequencies(
        int(rotary_dim), float(base), None if scaling is None else ctypes.byref(scaling), _host_addr(freq)))
    return freq


def sf_rotary_turns(freq) -> np.ndarray:
    """Frequencies as turns per position in units of 2^-64, whole turns left out (uint64)."""
    freq = np.ascontiguousarray(freq, dtype=np.float64)
    turns = np.empty(freq.shape, dtype=np.uint64)
    _check("sf_rotary_turns", lib().sf_rotary_turns(_host_addr(freq), freq.size, _host_addr(turns)))
    return turns


def _rows(t, name, shape):
    """Checks a bf16 tensor [T, H, D] whose tokens may lie apart; returns its token stride."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must live on the GPU (got {t.device})")
    if t.dtype is not torch.bfloat16:
        raise ValueError(f"{name} must be torch.bfloat16 (got {t.dtype})")
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    _, heads, d = shape
    if shape[0] > 1 and t.stride(0) < heads * d or t.stride(2) != 1 or (heads > 1 and t.stride(1) != d):
        raise ValueError(f"{name}: a token's heads must be contiguous, and tokens must not overlap")
    return t.stride(0) if shape[0] > 1 else heads * d


def _extent(t):
    """First byte of a tensor's elements and the one behind the last."""
    at = t.data_ptr()
    return at, at + (sum((n - 1) * s for n, s in zip(t.shape, t.stride())) + 1) * t.element_size() if t.numel() else at


def _overlap(a, b):
    (a0, a1), (b0, b1) = _extent(a), _extent(b)
    return a0 < b1 and b0 < a1 and not _interleaved(a, b)


def _check_turned(x, x_out, name, others):
    """An output is its input's own place, or overlaps none. (x among the others twice is read by another part of the
    call, too.)"""
    others = list(others)
    if x_out.data_ptr() == x.data_ptr() and x_out.stride() == x.stride():
        own = next((i for i, t in enumerate(others) if t is x), None)
        if own is not None:
            del others[own]
    if any(_overlap(x_out, t) for t in others):
        raise ValueError(f"{name} overlaps an input")


def _interleaved(a, b):
    """Whether two tensors [T, H, D] of one token stride lie in separate columns of the same rows."""
    if a.shape[0] <= 1 or a.stride(0) != b.stride(0):
        return False
    stride = a.stride(0)
    off = (b.data_ptr() - a.data_ptr()) // 2 % stride   # b's first column from a's
    nx, ny = a.shape[1] * a.shape[2], b.shape[1] * b.shape[2]
    return off >= nx and off + ny <= stride


def sf_rotary(rotary, turns, positions, q, k, q_out, k_out, stream=None):
    """Enqueues the turn of q and k (bf16 [T, H, D], parts of wider rows allowed, either may be None with its output) by
    positions (device int32 [T]). rotary: a sf_rotary_desc; turns: device int64 [rotary_dim / 2]."""
    t = positions.numel()
    _dev(positions, "positions", torch.int32, (t,))
    _dev(turns, "turns", torch.int64, (rotary.rotary_dim // 2,))
    args, heads = [], []
    for x, out, name in ((q, q_out, "q"), (k, k_out, "k")):
        if x is None:
            args += [None, 0, None, 0]
            heads.append(0)
            continue
        shape = (t, x.shape[1], rotary.head_dim)
        args += [x.data_ptr(), _rows(x, name, shape), out.data_ptr(), _rows(out, name + "_out", shape)]
        heads.append(x.shape[1])
    _check("sf_rotary", lib().sf_rotary(ctypes.byref(rotary), t, *heads, _addr(turns), _addr(positions), *args, _stream(stream)))


def sf_rotary_store_plan(desc, seq_lens, q_lens=None, first_pos=None, work_host=None):
    """Plans the turn and store of the last q_lens[s] of seq_lens[s] tokens (None: a decode step). Returns (info, work_host)."""
    n = desc.num_seqs
    lens, qls, first = (_host_i32(x, name, n) for x, name in ((seq_lens, "seq_lens"), (q_lens, "q_lens"), (first_pos, "first_pos")))
    info = sf_store_info()
    return _planned("sf_rotary_store_plan", info, lambda w, cap: lib().sf_rotary_store_plan(
        ctypes.byref(desc), _host_addr(lens), _addr(qls), _addr(first), w, cap, ctypes.byref(info)), work_host)


def sf_rotary_store(desc, rotary, info, work_host, work_dev, turns, q, q_out, k_new, v_new, new_pages, k_pool, v_pool,
                    block_table, stream=None):
    """Enqueues the turn of queries and keys and the store of keys and values into a bf16 cache. rotary: a sf_rotary_desc or
    None; q and q_out may be None; new_pages: device int32 [B] or None."""
    hq, hkv, d = desc.num_q_heads, desc.num_kv_heads, desc.head_dim
    rows = info.num_q_rows
    sk, sv = _rows(k_new, "k_new", (rows, hkv, d)), _rows(v_new, "v_new", (rows, hkv, d))
    sq, so = (0, 0) if q is None else (_rows(q, "q", (rows, hq, d)), _rows(q_out, "q_out", (rows, hq, d)))
    if new_pages is not None:
        _dev(new_pages, "new_pages", torch.int32, (desc.num_seqs,))
    if rotary is not None:
        _dev(turns, "turns", torch.int64, (rotary.rotary_dim // 2,))
    _check_pools(desc.num_pages, hkv, d, k_pool, v_pool, block_table, desc.num_seqs, None)
    _check_work(info, work_dev)
    _check("sf_rotary_store", lib().sf_rotary_store(
        ctypes.byref(desc), None if rotary is None else ctypes.byref(rotary), ctypes.byref(info), _addr(work_host),
        _addr(work_dev), _addr(turns), _addr(q), sq, _addr(q_out), so, _addr(k_new), sk, _addr(v_new), sv, _addr(new_pages),
        _addr(k_pool), _addr(v_pool), _addr(block_table), _stream(stream)))


_cus = {}


def _compute_units(index):
    if index not in _cus:
        _cus[index] = torch.cuda.get_device_properties(index).multi_processor_count
    return _cus[index]


class _SharedScratch:
    """Device memory for the partial results of cut plans, shared by the live
    ExtendAttention objects: one block per thread and stream. A thread's calls on
    one stream run one after the other, so each may overwrite what the last one
    left, and torch's allocator takes a dropped block back in that stream's order.
    At most BLOCKS blocks are kept (the least recently used goes first; an object
    that took it last keeps it until its next call), none once the last object is
    gone. Per-object memory would cost every new object
    of a process a device allocation (30 to 80 us) while others live."""
    BLOCKS = 4

    def __init__(self):
        self._lock = threading.RLock()   # a collection inside may drop an object
        self._blocks = {}   # (thread, device, stream) -> _Halves, least recently used first
        self.version = 0    # changes when blocks come and go
        self._live = 0
        self._dead = []     # runners of dropped objects, with what they lent
        self._capturing = torch.cuda.is_current_stream_capturing

    def join(self):
        with self._lock:
            self._live += 1

    def leave(self):
        with self._lock:
            self._live -= 1
            if self._live == 0:
                self._blocks.clear()
                self.version += 1

    def bury(self, destroy, runner, lent):
        """Destroys a dropped object's runner, which waits for its calls before what
        it lent may go. The wait would break a capture: then the next object sees to it."""
        with self._lock:
            self._dead.append((destroy, runner, lent))
        if not self._capturing():
            self.reap()

    def reap(self):
        while self._dead:
            with self._lock:
                dead = self._dead.pop() if self._dead else None
            if dead is not None:
                dead[0](dead[1])

    def get(self, key):
        """The block of (thread, device, stream), or None. It stands until `version` changes."""
        with self._lock:
            block = self._blocks.pop(key, None)
            if block is not None:
                self._blocks[key] = block
            return block

    def grow(self, key, nbytes):
        """Sees to a block whose halves have at least nbytes each."""
        with self._lock:
            self.version += 1
            block = self._blocks.pop(key, None)
            if block is None or block.nbytes < nbytes:
                block = None   # back to the allocator before the larger one is taken
                block = _Halves(torch.empty(2 * nbytes, dtype=torch.uint8, device=key[1]), nbytes)
            self._blocks[key] = block
            while len(self._blocks) > self.BLOCKS:
                del self._blocks[next(iter(self._blocks))]


class _Halves:
    """Device memory that calls in a row take one half of and then the other:
    partial results written where the call before was just read cost up to 2.3 us
    (5 sequences of up to 608 tokens 31.1 us a call in one place, 29.0 in two)."""

    def __init__(self, memory, nbytes):
        self.memory, self.nbytes, self.at = memory, nbytes, memory.data_ptr()

    def next(self):
        self.at = 2 * self.memory.data_ptr() + self.nbytes - self.at
        return self.at


_scratch = _SharedScratch()


class ExtendAttention:
    """Plans and launches extend attention for one batch of re-prefills.

    Each call goes through a native runner (sf_runner_extend): it plans into
    pinned memory that the launches read in place, so calls queue up behind
    each other without waiting. The pinned slots and the device memory for
    partial results are torch tensors that are lent to the runner: this object
    keeps the slots and up to 1 MiB of device memory, larger partial results (up
    to 256 MB) go to a block of twice the size that all live objects share. (A
    call with a `stream` argument keeps what it needs, as the block belongs to
    the current stream.) Where the device has no room for a cut plan's partial
    results, the call takes sf_extend_attn, whose plan needs only its own list.

    A stream that is being captured into a graph takes sf_extend_attn too, on a
    work list that the graph uploads at each replay. Captured calls share a list
    only where it is the same; none is rewritten or freed while the object lives,
    so the object must outlive the graphs. Pinned memory can't be allocated
    during a capture, so an eager call keeps room for its own batch's list: one
    that is captured after it allocates nothing."""

    def __init__(self, num_q_heads, num_kv_heads, head_dim, device=None):
        self.hq, self.hkv, self.d = int(num_q_heads), int(num_kv_heads), int(head_dim)
        self.device = torch.device("cuda") if device is None else torch.device(device)
        self._L = None
        self._runner = ctypes.c_void_p()
        self._memory = sf_runner_memory()
        self._lent = []         # what _memory lends for longer than a call; before it, what calls may still use
        self._at = self._block = None   # the shared block that it found, and where
        self._large = None      # a plan took the shared block (None: a new object looks for one)
        self._spare = [None, 0, None, 0, 0]   # pinned, device (offsets in bytes) and the bytes left for captured lists
        self._captured = []     # their lists (pinned, device), which graphs read
        self.last_info = None

    # What a new object lends: slots and device memory that hold most short
    # plans, so that its first call seldom has to ask and plan twice. First
    # calls, from call to result, 28/4 heads (us; in brackets with the plan of
    # whole items alone, in braces when every first call asked): 1000 tokens
    # 76 [95] {83}, 60 tokens 50 [58] {52}; with all earlier objects alive, whose
    # pinned memory torch cannot hand on, 145 [137] {190} and 100 [108] {96}.
    SLOTS, SLOT, DEVICE = 15, 1 << 15, 1 << 16
    KEEP = 1 << 20   # device bytes of a plan beyond which it takes the shared block

    def _create(self, stream):
        if self._L is None:
            L = lib()
            shape = make_desc(0, self.hq, self.hkv, self.d, 1, 0, 1.0)
            with contextlib.nullcontext() if self._ordered(None) else torch.cuda.device(self.device):
                opts = make_opts(num_cus=_compute_units(torch.cuda.current_device()))
                _check("sf_runner_create", L.sf_runner_create(ctypes.byref(shape), ctypes.byref(opts),
                                                              ctypes.byref(self._runner)))
            self._L, self._scratch = L, _scratch
            _scratch.join()
            _scratch.reap()
        self._lend(self.SLOT, self.DEVICE - self.SLOT, stream)

    def _lend(self, slot, device, stream):
        """Other memory for the runner. What it held stays alive until a call has
        waited for the calls that use it."""
        m = self._memory
        slots = self.SLOTS if slot <= 1 << 16 else 4
        # One slot more, on both sides, for captured calls: sf_extend_attn's
        # list has at most a row for each of the runner's.
        pinned = torch.empty((slots + 1) * slot, dtype=torch.uint8, pin_memory=True)
        work = torch.empty(device + slot, dtype=torch.uint8, device=self.device)
        self._spare = [pinned, slots * slot, work, device, slot]
        if stream is not None:   # the allocation is ordered on the current stream
            torch.cuda.current_stream(self.device).synchronize()
        m.pinned, m.pinned_bytes, m.slots = pinned.data_ptr(), slots * slot, slots
        m.device, m.device_bytes = work.data_ptr(), device
        self._lent.append((pinned, work))

    def _ordered(self, stream):
        """Whether the call's launches go to the stream that torch's allocator serves now."""
        return stream is None and (self.device.index is None or self.device.index == torch.cuda.current_device())

    def _grow(self, stream):
        """More memory, as the last call asked."""
        m = self._memory
        need = (int(m.need_device) * 5 // 4 + 4096 + 255) // 256 * 256
        slot, device = int(m.pinned_bytes) // m.slots, int(m.device_bytes)
        if need > self.KEEP and self._ordered(stream):
            self._large = True
            self._scratch.grow((threading.get_ident(), torch.cuda.current_device(), _stream(None)), need)
        else:
            device = max(device, need)
        if m.need_slot > slot:
            slot = (int(m.need_slot) * 5 // 4 + 1023) // 256 * 256
        if slot != int(m.pinned_bytes) // m.slots or device != m.device_bytes:
            self._lend(slot, device, stream)

    def _run(self, args, stream):
        """One sf_runner_extend, on the shared block where a plan has needed it."""
        m = self._memory
        block = None
        if self._large is not False and self._ordered(stream):
            at = (threading.get_ident(), torch.cuda.current_device(), args[13], self._scratch.version)
            if at != self._at:
                self._at, self._block = at, self._scratch.get(at[:3])
            block = self._block
        call = self._L.sf_runner_extend if len(args) == 15 else self._L.sf_runner_extend_fp8
        if block is None:
            st = call(*args)
        else:
            kept = m.device, m.device_bytes
            m.device, m.device_bytes, m.device_per_call = block.next(), block.nbytes, 1
            st = call(*args)
            m.device, m.device_bytes, m.device_per_call = *kept, 0
        if self._large is None:
            self._large = m.need_device > m.device_bytes
            if not self._large:
                self._at = self._block = None
        if len(self._lent) > 1 and st in (0, CAPACITY):   # other slots: calls on what was lent before have been waited for
            del self._lent[:-1]
        return st

    def __call__(self, q, k_pool, v_pool, block_table, seq_lens, q_lens, scale, out=None, lse=None,
                 k_new=None, v_new=None, stream=None, fp8=None):
        """fp8 = (k_scale, v_scale): k_pool and v_pool are an fp8 cache, which k_new and v_new are stored into by
        sf_kv_store_fp8's rule, and out may be bf16."""
        lens = np.ascontiguousarray(np.asarray(seq_lens), dtype=np.int32)
        qls = np.ascontiguousarray(np.asarray(q_lens), dtype=np.int32)
        if lens.ndim != 1 or lens.shape != qls.shape:
            raise ValueError("seq_lens and q_lens must have num_seqs entries")
        desc = make_desc(lens.size, self.hq, self.hkv, self.d, block_table.shape[1], k_pool.shape[0], scale)
        rows = int(qls.sum())
        if DEBUG_CHECKS:
            check_block_table(desc, block_table, np.where(qls > 0, lens, 0))
        if out is None:
            with _made_on(stream, self.device):
                out = torch.empty((rows, self.hq, self.d), dtype=torch.float32, device=self.device)
        _check_extend(desc, rows, q, k_pool, v_pool, block_table, out, lse, k_new, v_new, fp8)
        info = sf_extend_info()
        tensors = (q, k_pool, v_pool, block_table, out, lse, k_new, v_new, fp8)
        try:
            if not self._lent:
                if torch.cuda.is_current_stream_capturing():   # nothing is created in a capture
                    self.last_info = self._call_captured(desc, lens, qls, tensors, stream)
                    return out
                self._create(stream)
            args = (self._runner, ctypes.byref(desc), _host_addr(lens), _host_addr(qls), q.data_ptr(), _addr(k_new),
                    _addr(v_new), k_pool.data_ptr(), v_pool.data_ptr(), block_table.data_ptr(), out.data_ptr(), _addr(lse),
                    ctypes.byref(self._memory), _stream(stream), ctypes.byref(info))
            if fp8 is not None:
                args += (fp8[0].data_ptr(), fp8[1].data_ptr(), int(out.dtype is torch.bfloat16))
            st = self._run(args, stream)
            if st == CAPACITY:
                self._grow(stream)
                st = self._run(args, stream)
        except torch.OutOfMemoryError:
            st = CAPACITY
        if st == CAPACITY:
            self.last_info = self._call_whole(desc, lens, qls, tensors, stream)
            return out
        if st == UNSUPPORTED:
            info = self._call_captured(desc, lens, qls, tensors, stream)
        else:
            _check("sf_runner_extend", st)
            need = info.work_bytes
            if fp8 is not None:   # a captured call takes the store's list, too, which the runner's plan holds
                need = max(need, int(self._memory.need_slot))
            if self._spare[4] < need:   # captured calls took it
                self._spare = self._room(need)
        self.last_info = info
        return out

    def _room(self, nbytes):
        return [torch.empty(nbytes, dtype=torch.uint8, pin_memory=True), 0,
                torch.empty(nbytes, dtype=torch.uint8, device=self.device), 0, nbytes]

    def _captured_list(self, work):
        """(pinned, device) lists with the rows of `work`, of this object's captured calls alone."""
        for host, dev in self._captured:
            if host.numel() == work.size and np.array_equal(host.numpy(), work):
                return host, dev
        if self._spare[4] < work.nbytes:
            try:
                self._spare = self._room(work.nbytes)
            except RuntimeError as e:
                raise RuntimeError("no room for a captured extend call's work list: make an eager call with this batch "
                                   "before the capture") from e
        pinned, p, device, d, left = self._spare
        host, dev = (t[at: at + work.nbytes].view(torch.int32) for t, at in ((pinned, p), (device, d)))
        self._spare = [pinned, p + work.nbytes, device, d + work.nbytes, left - work.nbytes]
        host.numpy()[:] = work
        self._captured.append((host, dev))
        return host, dev

    def _launch_whole(self, desc, lens, qls, tensors, stream, lists):
        """sf_extend_attn, or the store and sf_extend_attn_fp8, on lists(work list) -> (pinned or None, device)."""
        info, work = sf_extend_attn_plan(desc, lens, qls)
        if info.num_items == 0:
            return info
        fp8 = tensors[-1]
        if fp8 is None:
            sf_extend_attn(desc, info, *lists(work[: info.work_bytes // 4]), *tensors[:-1], stream=stream)
            return info
        q, k_pool, v_pool, block_table, out, lse, k_new, v_new = tensors[:-1]
        if k_new is not None:
            sinfo, rows = sf_kv_store_fp8_plan(desc, lens, qls)
            sf_kv_store_fp8(desc, sinfo, *lists(rows[: sinfo.work_bytes // 4]), k_new, v_new, None, k_pool, v_pool, *fp8,
                            block_table, stream=stream)
        sf_extend_attn_fp8(desc, info, *lists(work[: info.work_bytes // 4]), q, k_pool, v_pool, *fp8, block_table, out,
                           lse, stream=stream)
        return info

    def _call_captured(self, desc, lens, qls, tensors, stream):
        return self._launch_whole(desc, lens, qls, tensors, stream, self._captured_list)

    def _call_whole(self, desc, lens, qls, tensors, stream):
        kept = []

        def lists(work):
            kept.append(torch.from_numpy(work).to(self.device))   # uploaded when this returns
            return None, kept[-1]

        info = self._launch_whole(desc, lens, qls, tensors, stream, lists)
        if stream is not None:   # the lists belong to the current stream
            torch.cuda.ExternalStream(_stream(stream), device=self.device).synchronize()
        return info

    def __del__(self):
        r = getattr(self, "_runner", None)
        if r is not None and r.value:
            self._scratch.bury(self._L.sf_runner_destroy, r.value, self._lent)
            r.value = None
            self._scratch.leave()


class PagePool:
    """The library's host page allocator (LIFO free list over page ids)."""

    def __init__(self, num_pages: int):
        self._p = ctypes.c_void_p()
        self._L = lib()
        _check("sf_page_pool_create", self._L.sf_page_pool_create(int(num_pages), ctypes.byref(self._p)))
        self.num_pages = int(num_pages)

    def available(self) -> int:
        return int(self._L.sf_page_pool_available(self._p))

    def claim(self, pages) -> None:
        a = np.ascontiguousarray(pages, dtype=np.int32)
        _check("sf_page_pool_claim", self._L.sf_page_pool_claim(self._p, a.ctypes.data, a.size))

    def alloc(self, n: int) -> np.ndarray:
        out = np.empty(max(0, int(n)), dtype=np.int32)
        _check("sf_page_pool_alloc", self._L.sf_page_pool_alloc(self._p, int(n), out.ctypes.data))
        return out

    def share(self, pages) -> None:
        """One more holder for every page listed."""
        a = np.ascontiguousarray(pages, dtype=np.int32)
        _check("sf_page_pool_share", self._L.sf_page_pool_share(self._p, a.ctypes.data, a.size))

    def release(self, pages) -> None:
        a = np.ascontiguousarray(pages, dtype=np.int32)
        _check("sf_page_pool_release", self._L.sf_page_pool_release(self._p, a.ctypes.data, a.size))

    def __del__(self):
        p = getattr(self, "_p", None)
        if p is not None and p.value:
            self._L.sf_page_pool_destroy(p)
        self._p = None


def cost_throughput(model: sf_cost_model, state: sf_instance_state) -> float:
    return float(lib().sf_cost_throughput(ctypes.byref(model), ctypes.byref(state)))


def cost_marginal_gain(model: sf_cost_model, state: sf_instance_state, length: float) -> float:
    return float(lib().sf_cost_marginal_gain(ctypes.byref(model), ctypes.byref(state), float(length)))


def cost_ideal_gain(model: sf_cost_model, length: float) -> float:
    return float(lib().sf_cost_ideal_gain(ctypes.byref(model), float(length)))


def route(model: sf_cost_model, mu: float, min_initial_version: int, instances, trajectories):
    """sf_route on objects with version/running/waiting/kv (instances) and
    version (None = initial)/length (trajectories). Returns (targets, the
    updated instances as sf_instance_state)."""
    ni, nt = len(instances), len(trajectories)
    inst = (sf_instance_state * max(1, ni))()
    for i, s in enumerate(instances):
        inst[i] = sf_instance_state(int(s.version), int(s.running), int(s.waiting), 0, float(s.kv))
    tr = (sf_trajectory * max(1, nt))()
    for j, t in enumerate(trajectories):
        tr[j] = sf_trajectory(-1 if t.version is None else int(t.version), 0, float(t.length))
    target = np.full(max(1, nt), -1, dtype=np.int32)
    routed = ctypes.c_int32()
    _check("sf_route", lib().sf_route(ctypes.byref(model), float(mu), int(min_initial_version), inst, ni, tr, nt,
                                      target.ctypes.data, ctypes.byref(routed)))
    after = [_InstanceView(inst[i]) for i in range(ni)]
    return target[:nt].tolist(), after


class _InstanceView:
    def __init__(self, s: sf_instance_state):
        self.version, self.running, self.waiting, self.kv = s.version, s.num_running, s.num_waiting, s.kv_cache


def sf_decode_attn_combine(desc, info, work_dev, workspace, out, lse=None, stream=None):
    """Enqueues the log-sum-exp merge of split sequences (no-op if none)."""
    if info.num_combine == 0:
        return
    _dev(out, "out", torch.float32, (desc.num_seqs, desc.num_q_heads, desc.head_dim))
    _dev(work_dev, "work_dev", torch.int32)
    _dev(workspace, "workspace", workspace.dtype)
    if lse is not None:
        _dev(lse, "lse", torch.float32, (desc.num_seqs, desc.num_q_heads))
    _check("sf_decode_attn_combine", lib().sf_decode_attn_combine(
        ctypes.byref(desc), ctypes.byref(info), _addr(work_dev), _addr(workspace),
        workspace.numel() * workspace.element_size(), _addr(out), _addr(lse), _stream(stream)))


SCRATCH_BYTES = 32 << 20   # SF_SCRATCH_BYTES of the header


def sf_decode_attn_scratch(desc, info, work_dev, q, k_pool, v_pool, block_table, out, lse=None, stream=None):
    """sf_decode_attn + sf_decode_attn_combine with the partials in the
    library's own device array (allocates nothing). work_dev: the plan,
    already on the device."""
    b, hq, hkv, d = desc.num_seqs, desc.num_q_heads, desc.num_kv_heads, desc.head_dim
    _dev(q, "q", torch.bfloat16, (b, hq, d))
    _dev(k_pool, "k_pool", torch.bfloat16, (desc.num_pages, hkv, d // 8, PAGE, 8))
    _dev(v_pool, "v_pool", torch.bfloat16, (desc.num_pages, hkv, d, PAGE))
    _dev(block_table, "block_table", torch.int32, (b, desc.block_table_stride))
    _dev(out, "out", torch.float32, (b, hq, d))
    _dev(work_dev, "work_dev", torch.int32)
    if work_dev.numel() * 4 < info.work_bytes:
        raise ValueError("work_dev is smaller than the plan")
    if lse is not None:
        _dev(lse, "lse", torch.float32, (b, hq))
    _check("sf_decode_attn_scratch", lib().sf_decode_attn_scratch(
        ctypes.byref(desc), ctypes.byref(info), _addr(work_dev), _addr(q), _addr(k_pool), _addr(v_pool),
        _addr(block_table), _addr(out), _addr(lse), _stream(stream)))


def kernel_event(ev, stream):
    """The hipEvent_t behind a torch timing event, for an entry point that
    records the kernel's own start or end time into it. torch creates an
    event on its first record, so a fresh one is recorded on `stream` once."""
    if ev.cuda_event == 0:
        ev.record(stream)
    return ev.cuda_event


def sf_debug_stream_read(buf, sink, blocks=16384, stream=None, events=None):
    """Reads every byte of the uint8 device tensor buf once (measurement
    support); sink: a uint8 device tensor of at least 16 bytes. events, if
    given, is a (start, end) pair of torch timing events that take the
    kernel's own start and end times."""
    _dev(buf, "buf", torch.uint8)
    _dev(sink, "sink", torch.uint8)
    if sink.numel() * sink.element_size() < 16:
        raise ValueError("sink must hold at least 16 bytes")
    s = stream or torch.cuda.current_stream(buf.device)
    ev = (None, None) if events is None else (kernel_event(events[0], s), kernel_event(events[1], s))
    _check("sf_debug_stream_read", lib().sf_debug_stream_read(
        _addr(buf), buf.numel() * buf.element_size(), _addr(sink), int(blocks), s.cuda_stream, *ev))


def sf_debug_gather_kv(desc, k_pool, v_pool, block_table, seq, kv_head, length, k_dense, v_dense,
                       stream=None):
    """Dense [length, D] bf16 copies of one (sequence, KV head) via the kernel's translation."""
    d = desc.head_dim
    _dev(k_pool, "k_pool", torch.bfloat16)
    _dev(v_pool, "v_pool", torch.bfloat16)
    _dev(block_table, "block_table", torch.int32)
    _dev(k_dense, "k_dense", torch.bfloat16, (length, d))
    _dev(v_dense, "v_dense", torch.bfloat16, (length, d))
    _check("sf_debug_gather_kv", lib().sf_debug_gather_kv(
        ctypes.byref(desc), _addr(k_pool), _addr(v_pool), _addr(block_table), int(seq),
        int(kv_head), int(length), _addr(k_dense), _addr(v_dense), _stream(stream)))


# ----------------------------------------------------------------------------
# convenience runner: owns the pinned work-list ring and the device buffers
# ----------------------------------------------------------------------------
class DecodeAttention:
    """Plan + attention + combine for successive decode steps, through the
    library's native runner (sf_runner_create / sf_runner_step): one call per
    step plans into the runner's pinned, device-mapped ring and launches the
    kernels, which read that work list in place, on the caller's stream (a call on another stream than
    the last one waits there for the calls before it: they share a workspace). A cache's
    tensors are checked once (the first 256 sets are remembered while they live)."""

    def __init__(self, num_q_heads, num_kv_heads, head_dim, device=None, num_cus=None,
                 opts: sf_plan_opts | None = None):
        self.hq, self.hkv, self.d = int(num_q_heads), int(num_kv_heads), int(head_dim)
        self.device = torch.device(device or "cuda")
        if num_cus is None:
            num_cus = torch.cuda.get_device_properties(self.device).multi_processor_count
        self.opts = opts if opts is not None else make_opts(num_cus=num_cus)
        if self.opts.num_cus == 0:
            self.opts.num_cus = num_cus
        self.L = lib()
        self._runners = {}
        self._info = sf_plan_info()
        self._info_ref = ctypes.byref(self._info)
        self._extras, self._fp8_only = sf_runner_extras(), sf_runner_extras()
        self._extras_ref, self._fp8_only_ref = ctypes.byref(self._extras), ctypes.byref(self._fp8_only)
        self._checked = {}
        self._checks_left = 256   # views made anew for every call are never known: then nothing is remembered
        self._desc_key = None
        self._desc = self._desc_ref = None
        self._stepped = False
        self._lse, self._old_lse = None, []
        self._host_checked = False   # set by a caller that checked its own host copy

    def _runner(self, chunk_pages):
        o = self.opts
        key = (o.num_cus, int(chunk_pages or 0), o.workers_per_cu, o.min_chunk_pages, o.xcd_parity_skew)
        r = self._runners.get(key)
        if r is None:
            opts = sf_plan_opts(*key)
            shape = make_desc(0, self.hq, self.hkv, self.d, 1, 0, 1.0)
            r = ctypes.c_void_p()
            with torch.cuda.device(self.device):
                _check("sf_runner_create", self.L.sf_runner_create(ctypes.byref(shape), ctypes.byref(opts),
                                                                   ctypes.byref(r)))
            self._runners[key] = r
        return r

    def _check_tensors(self, q, k_pool, v_pool, block_table, out, lse, fp8=None):
        hkv, d, b = self.hkv, self.d, q.shape[0]
        _dev(q, "q", torch.bfloat16, (b, self.hq, d))
        _dev(out, "out", torch.float32, (b, self.hq, d))
        if lse is not None:
            _dev(lse, "lse", torch.float32, (b, self.hq))
        ks, vs = (None, None) if fp8 is None else fp8
        remember = self._checks_left > 0
        if remember:
            key = (b, id(k_pool), id(v_pool), id(block_table), id(ks), id(vs))
            known = self._checked.get(key)
            if known is not None and known[0]() is k_pool and known[1]() is v_pool and known[2]() is block_table and \
                    (fp8 is None or (known[3]() is ks and known[4]() is vs)):
                return
        n = k_pool.shape[0]
        if fp8 is None:
            _dev(k_pool, "k_pool", torch.bfloat16, (n, hkv, d // 8, PAGE, 8))
            _dev(v_pool, "v_pool", torch.bfloat16, (n, hkv, d, PAGE))
        else:
            _dev(k_pool, "k_pool8", torch.uint8, (n, hkv, PAGE * d))
            _dev(v_pool, "v_pool8", torch.uint8, (n, hkv, PAGE * d))
            _dev(ks, "k_scale", torch.float32, (n, hkv))
            _dev(vs, "v_scale", torch.float32, (n, hkv))
        _dev(block_table, "block_table", torch.int32, (b, block_table.shape[1]))
        if remember:
            self._checks_left -= 1
            self._checked[key] = [weakref.ref(t) for t in (k_pool, v_pool, block_table, ks, vs) if t is not None]

    def reserve(self, seq_lens, num_pages, block_table_stride, chunk_pages=None, fp8=False, stream=None):
        """Sizes the native runner's workspace and work-list ring for a step
        over seq_lens (the largest batch to come) ahead of the steps, so no
        step stalls to grow them (sf_runner_reserve_batch): steps of any kind,
        over these sequences, with up to twice the pages, or over fewer or
        shorter ones."""
        lens = np.ascontiguousarray(seq_lens, dtype=np.int32)
        desc = make_desc(lens.size, self.hq, self.hkv, self.d, block_table_stride, num_pages, 1.0)
        o = self.opts
        opts = sf_plan_opts(o.num_cus, int(chunk_pages or 0), o.workers_per_cu, o.min_chunk_pages, o.xcd_parity_skew)
        info = sf_plan_info()
        st = self.L.sf_runner_plan(ctypes.byref(desc), lens.ctypes.data, ctypes.byref(opts), int(bool(fp8)), None, 0,
                                   ctypes.byref(info))
        _check("sf_runner_plan", st)
        main = stream or torch.cuda.current_stream(self.device)
        with torch.cuda.device(self.device):
            _check("sf_runner_reserve_batch", self.L.sf_runner_reserve_batch(self._runner(chunk_pages), lens.ctypes.data,
                                                                             lens.size, main.cuda_stream))

    def __call__(self, q, k_pool, v_pool, block_table, seq_lens, scale, out=None, lse=None,
                 chunk_pages=None, stream: torch.cuda.Stream | None = None, attn_events=None,
                 append=None, fp8=None):
        """One decode step on `stream` (default: the current stream). attn_events,
        if given, is a (start, end) pair of torch timing events that take the
        attention kernel's own start and end times (none if the step launches
        no attention kernel). append = (k_new, v_new, new_pages) makes it an
        append-then-attend step: k_new, v_new are device bf16 [B, Hkv, D] and
        new_pages a host int32 [B] array (-1 = the token's page is already
        held), uploaded together with the work list. fp8 = (k_scale, v_scale)
        makes k_pool / v_pool an fp8 cache (uint8 E4M3 codes [N, Hkv, 16*D],
        fp32 scales [N, Hkv]). With both, the newest tokens are stored first
        (sf_kv_store_fp8's rule) and attended as stored."""
        b = q.shape[0]
        main = stream.cuda_stream if stream else _current_stream(self.device)
        if out is None:
            with _made_on(stream, self.device):
                out = torch.empty((b, self.hq, self.d), dtype=torch.float32, device=self.device)
        self._check_tensors(q, k_pool, v_pool, block_table, out, lse, fp8)
        dkey = (b, block_table.shape[1], k_pool.shape[0], float(scale))
        if dkey != self._desc_key:
            self._desc = make_desc(b, self.hq, self.hkv, self.d, block_table.shape[1], k_pool.shape[0], scale)
            self._desc_ref = ctypes.byref(self._desc)
            self._desc_key = dkey
        if isinstance(seq_lens, torch.Tensor):
            seq_lens = seq_lens.cpu().numpy()
        lens = seq_lens if (isinstance(seq_lens, np.ndarray) and seq_lens.dtype == np.int32
                            and seq_lens.flags.c_contiguous) else np.ascontiguousarray(seq_lens, np.int32)
        if lens.shape != (b,):
            raise ValueError("seq_lens must have one entry per sequence")
        # A plain step has no extras, one over an fp8 cache only the scales.
        extras = None
        if append is not None or attn_events is not None:
            ex, extras = self._extras, self._extras_ref
            ex.k_new = ex.v_new = ex.new_pages_host = ex.k_scale = ex.v_scale = ex.attn_start = ex.attn_end = None
        elif fp8 is not None:
            ex, extras = self._fp8_only, self._fp8_only_ref
        pages = None
        if append is not None:
            k_new, v_new, new_pages = append
            _dev(k_new, "k_new", torch.bfloat16, (b, self.hkv, self.d))
            _dev(v_new, "v_new", torch.bfloat16, (b, self.hkv, self.d))
            pages = np.ascontiguousarray(new_pages, dtype=np.int32)
            if pages.shape != (b,):
                raise ValueError("new_pages must have one entry per sequence")
            ex.k_new, ex.v_new, ex.new_pages_host = k_new.data_ptr(), v_new.data_ptr(), _host_addr(pages)
            if lse is None and fp8 is None:  # the merge reads lse back: keep one of our own
                if self._lse is None or self._lse.numel() < b * self.hq:
                    self._old_lse.append(self._lse)   # calls on other streams may still write it
                    with _made_on(stream, self.device):
                        self._lse = torch.empty(b * self.hq * 5 // 4 + 64, dtype=torch.float32, device=self.device)
                lse = self._lse[: b * self.hq].view(b, self.hq)
        if fp8 is not None:
            ex.k_scale, ex.v_scale = fp8[0].data_ptr(), fp8[1].data_ptr()
        if DEBUG_CHECKS and not self._host_checked:
            # an appending step reads the pool for its L - 1 cached tokens only
            # (the newest token's page may still be -1: the step writes it)
            check_block_table(self._desc, block_table, lens - 1 if append is not None else lens)
            if pages is not None and np.any((pages < -1) | (pages >= k_pool.shape[0])):
                raise ValueError("new_pages holds a page id outside the pool")
        self._host_checked = False
        if attn_events is not None:
            timed = stream or torch.cuda.current_stream(self.device)
            ex.attn_start = kernel_event(attn_events[0], timed)
            ex.attn_end = kernel_event(attn_events[1], timed)
        _check("sf_runner_step", self.L.sf_runner_step(
            self._runner(chunk_pages), self._desc_ref, _host_addr(lens), q.data_ptr(), k_pool.data_ptr(),
            v_pool.data_ptr(), block_table.data_ptr(), out.data_ptr(), None if lse is None else lse.data_ptr(),
            extras, main, self._info_ref))
        self._stepped = True
        return out

    @property
    def last_info(self):
        """A copy of the last step's plan; None before the first."""
        return sf_plan_info.from_buffer_copy(self._info) if self._stepped else None

    def _call_desc(self, k_pool, block_table, seq_lens, scale):
        """(desc, lengths) of a call besides the steps."""
        lens = _host_i32(seq_lens, "seq_lens", block_table.shape[0])
        desc = make_desc(lens.size, self.hq, self.hkv, self.d, block_table.shape[1], k_pool.shape[0], scale)
        return desc, lens

    def store_fp8(self, k_new, v_new, k_pool8, v_pool8, fp8, block_table, seq_lens, q_lens, new_pages=None, stream=None):
        """Stores the last q_lens[s] of seq_lens[s] tokens (k_new, v_new: bf16 [T, Hkv, D]) into an fp8 cache, fp8 =
        (k_scale, v_scale), through the runner (sf_runner_store_fp8). new_pages: host int32 [B], the page of a
        sequence's last token where that opens one, else -1; None: every page is in the block table."""
        desc, lens = self._call_desc(k_pool8, block_table, seq_lens, 1.0)
        qls, pages = _host_i32(q_lens, "q_lens", lens.size), _host_i32(new_pages, "new_pages", lens.size)
        rows = int(qls.sum())
        _dev(k_new, "k_new", torch.bfloat16, (rows, self.hkv, self.d))
        _dev(v_new, "v_new", torch.bfloat16, (rows, self.hkv, self.d))
        _check_pools(desc.num_pages, self.hkv, self.d, k_pool8, v_pool8, block_table, lens.size, fp8)
        if DEBUG_CHECKS:
            _check_stored_pages(desc, block_table, lens, qls, pages)
        _check("sf_runner_store_fp8", self.L.sf_runner_store_fp8(
            self._runner(None), ctypes.byref(desc), _host_addr(lens), _host_addr(qls), k_new.data_ptr(), v_new.data_ptr(),
            _addr(pages), k_pool8.data_ptr(), v_pool8.data_ptr(), fp8[0].data_ptr(), fp8[1].data_ptr(),
            block_table.data_ptr(), stream.cuda_stream if stream else _current_stream(self.device)))

    def key_weights(self, q, lse, k_pool, block_table, seq_lens, q_lens, scale, weights, weights_out=None,
                    positions=None, held_lens=None, first_pos=None, k_scale=None, stream=None):
        """Adds every cached key's attention weight, summed over the query rows of the last q_lens[s] of seq_lens[s]
        tokens and over the heads of its group, to weights (sf_key_weights, through the runner)."""
        weights_out = weights if weights_out is None else weights_out
        desc, lens = self._call_desc(k_pool, block_table, seq_lens, scale)
        n = lens.size
        qls, held, pos = (_host_i32(x, name, n) for x, name in ((q_lens, "q_lens"), (held_lens, "held_lens"),
                                                                (first_pos, "first_pos")))
        rows = int(qls.sum())
        _dev(q, "q", torch.bfloat16, (rows, self.hq, self.d))
        _dev(lse, "lse", torch.float32, (rows, self.hq))
        _check_pools(desc.num_pages, self.hkv, self.d, k_pool, None, block_table, n, None if k_scale is None else (k_scale,))
        _check_slots(desc.num_pages, self.hkv, weights, weights_out, positions)
        if DEBUG_CHECKS:
            check_block_table(desc, block_table, np.where(qls > 0, lens, 0))
        _check("sf_runner_key_weights", self.L.sf_runner_key_weights(
            self._runner(None), ctypes.byref(desc), _host_addr(lens), _host_addr(qls), _addr(held), _addr(pos), q.data_ptr(),
            lse.data_ptr(), k_pool.data_ptr(), _addr(k_scale), block_table.data_ptr(), weights.data_ptr(),
            weights_out.data_ptr(), _addr(positions), stream.cuda_stream if stream else _current_stream(self.device)))

    def evict(self, k_pool, v_pool, block_table, seq_lens, keep_lens, weights, positions, weights_out=None,
              positions_out=None, ends=None, sinks=0, recent=0, fp8=None, stream=None):
        """Evicts down to at most keep_lens[s] tokens per (sequence, KV head) (sf_kv_evict, through the runner): the
        positions below `sinks` and the last `recent` before ends[s] (default: seq_lens) stay, then the heaviest."""
        weights_out = weights if weights_out is None else weights_out
        positions_out = positions if positions_out is None else positions_out
        desc, lens = self._call_desc(k_pool, block_table, seq_lens, 1.0)
        keep, end = _host_i32(keep_lens, "keep_lens", lens.size), _host_i32(ends, "ends", lens.size)
        _check_pools(desc.num_pages, self.hkv, self.d, k_pool, v_pool, block_table, lens.size, fp8)
        _check_slots(desc.num_pages, self.hkv, weights, weights_out, positions, positions_out)
        if DEBUG_CHECKS:
            check_block_table(desc, block_table, lens)
        k_scale, v_scale = fp8 if fp8 is not None else (None, None)
        _check("sf_runner_evict", self.L.sf_runner_evict(
            self._runner(None), ctypes.byref(desc), _host_addr(lens), _host_addr(keep), _addr(end), int(sinks), int(recent),
            k_pool.data_ptr(), v_pool.data_ptr(), _addr(k_scale), _addr(v_scale), block_table.data_ptr(), weights.data_ptr(),
            positions.data_ptr(), weights_out.data_ptr(), positions_out.data_ptr(),
            stream.cuda_stream if stream else _current_stream(self.device)))

    def shared(self, q, k_pool, v_pool, block_table, seq_lens, group_offsets, shared_lens, scale, out=None, lse=None,
               fp8=None, stream=None):
        """One decode step of groups that share their first tokens (sf_shared_attn, through the runner): sequences
        group_offsets[i] .. group_offsets[i+1] - 1 hold shared_lens[i] common tokens in the pages that their block tables
        start with (host int32 arrays). The result is the plain step's over each sequence's seq_lens[s] tokens. out: fp32
        (default) or bf16 [B, Hq, D]; fp8 = (k_scale, v_scale) of an fp8 cache."""
        if out is None:
            with _made_on(stream, self.device):
                out = torch.empty((q.shape[0], self.hq, self.d), dtype=torch.float32, device=self.device)
        desc, lens = self._call_desc(k_pool, block_table, seq_lens, scale)
        lens, offsets, shared = _host_groups(lens.size, lens, group_offsets, shared_lens)
        _check_step(desc, q, k_pool, v_pool, block_table, out, lse, fp8)
        if DEBUG_CHECKS and not self._host_checked:
            _check_group_pages(desc, block_table, lens, offsets, shared)
        self._host_checked = False
        k_scale, v_scale = fp8 if fp8 is not None else (None, None)
        _check("sf_runner_shared", self.L.sf_runner_shared(
            self._runner(None), ctypes.byref(desc), _host_addr(lens), shared.size, _host_addr(offsets), _host_addr(shared),
            q.data_ptr(), k_pool.data_ptr(), v_pool.data_ptr(), _addr(k_scale), _addr(v_scale), block_table.data_ptr(),
            out.data_ptr(), int(out.dtype is torch.bfloat16), _addr(lse),
            stream.cuda_stream if stream else _current_stream(self.device)))
        return out

    def rotate_store(self, rotary, q, k_new, v_new, k_pool, v_pool, block_table, seq_lens, q_lens=None, first_pos=None,
                     new_pages=None, q_out=None, stream=None):
        """Turns the queries and keys of the last q_lens[s] of seq_lens[s] tokens by their positions and stores the turned
        keys and the values into the pages of a bf16 cache (sf_rotary_store, through the runner). rotary: a Rotary, or
        None (nothing turns); q, k_new, v_new: bf16 [T, H, D], parts of wider rows allowed (q may be None). q_lens None is
        a decode step: a row per sequence, of which the running ones' (seq_lens[s] > 0) last token is new (the others' rows
        of q_out are not written). first_pos: host int32 [B], the first new token's position (default: its index in the
        cache); new_pages as in store_fp8. Returns the turned queries: q_out (may be q), by default a new tensor."""
        desc, lens = self._call_desc(k_pool, block_table, seq_lens, 1.0)
        n = lens.size
        qls, first, pages = (_host_i32(x, name, n) for x, name in ((q_lens, "q_lens"), (first_pos, "first_pos"),
                                                                   (new_pages, "new_pages")))
        rope, turns = None, None
        if rotary is not None:
            if rotary.head_dim != self.d:
                raise ValueError(f"rotary turns heads of {rotary.head_dim} dims, not {self.d}")
            rope, turns = rotary.desc_ref, rotary.turns_on(k_pool.device).data_ptr()
        rows = n if qls is None else int(qls.sum(dtype=np.int64))
        sk, sv = _rows(k_new, "k_new", (rows, self.hkv, self.d)), _rows(v_new, "v_new", (rows, self.hkv, self.d))
        sq = so = 0
        if q is not None:
            sq = _rows(q, "q", (rows, self.hq, self.d))
            if q_out is None:
                with torch.cuda.stream(stream):   # the stream that it is written on
                    q_out = torch.empty((rows, self.hq, self.d), dtype=torch.bfloat16, device=q.device)
            so = _rows(q_out, "q_out", (rows, self.hq, self.d))
            _check_turned(q, q_out, "q_out", [q, k_new, v_new])
        elif q_out is not None:
            raise ValueError("q_out without q")
        _check_pools(desc.num_pages, self.hkv, self.d, k_pool, v_pool, block_table, n, None)
        if DEBUG_CHECKS and not self._host_checked:
            _check_stored_pages(desc, block_table, lens, (lens > 0).astype(np.int32) if qls is None else qls, pages)
        self._host_checked = False
        _check("sf_runner_rotary_store", self.L.sf_runner_rotary_store(
            self._runner(None), ctypes.byref(desc), rope, _host_addr(lens), _addr(qls), _addr(first), turns, _addr(q), sq,
            _addr(q_out), so, k_new.data_ptr(), sk, v_new.data_ptr(), sv, _addr(pages), k_pool.data_ptr(),
            v_pool.data_ptr(), block_table.data_ptr(), stream.cuda_stream if stream else _current_stream(self.device)))
        return q_out

    def __del__(self):
        L = getattr(self, "L", None)
        for r in getattr(self, "_runners", {}).values():
            if L is not None and r.value:
                L.sf_runner_destroy(r)
        self._runners = {}


class Rotary:
    """Rotary positions: turns queries and keys by their positions (sf_rotary). The first rotary_dim dims of a head
    (default: all) turn, in pairs half of rotary_dim apart (layout "half") or of neighbours ("interleaved"), by
    angles of position * freq[i]; freq (radians per position, float64 [rotary_dim / 2]) defaults to base^(-2i / rotary_dim).
    scaling: a dict for contexts longer than the trained one, with factor and, for frequencies that keep their turns in it,
    original (tokens), low, high (turns; sf_rotary_scaling); its magnitude (default 1) multiplies what is turned. Its ramp is
    linear in the turns; frequencies of a ramp in the pair's index, as some configurations have it, go in as freq."""

    def __init__(self, head_dim, rotary_dim=None, base=10000.0, layout="half", scaling=None, freq=None, device=None):
        self.head_dim = int(head_dim)
        self.rotary_dim = self.head_dim if rotary_dim is None else int(rotary_dim)
        if layout not in ("half", "interleaved"):
            raise ValueError('layout must be "half" or "interleaved"')
        scaling = dict(scaling or {})
        magnitude = float(scaling.pop("magnitude", 1.0))
        if freq is None:
            c = None
            if scaling:
                c = sf_rotary_scaling(float(scaling.pop("factor")), float(scaling.pop("original", 0.0)),
                                      float(scaling.pop("low", 1.0)), float(scaling.pop("high", 4.0)))
            freq = sf_rotary_frequencies(self.rotary_dim, base, c)
        if scaling:
            raise ValueError(f"unknown scaling: {sorted(scaling)}")
        self.freq = np.ascontiguousarray(freq, dtype=np.float64)
        if self.freq.shape != (self.rotary_dim // 2,):
            raise ValueError("freq must have rotary_dim / 2 entries")
        self.desc = sf_rotary_desc(self.head_dim, self.rotary_dim, int(layout == "interleaved"), magnitude)
        self.desc_ref = ctypes.byref(self.desc)
        self._turns = torch.from_numpy(sf_rotary_turns(self.freq).view(np.int64))
        self._on = {}
        # an error of the arguments, if any, here and not at the first call
        _check("sf_rotary", lib().sf_rotary(self.desc_ref, 0, 0, 0, None, None, None, 0, None, 0, None, 0, None, 0, None))
        if device is not None:
            self.turns_on(torch.device(device))

    def turns_on(self, device):
        """The turns per position as a tensor on the device (uploaded at the first call there)."""
        index = torch.cuda.current_device() if device.index is None else device.index   # "cuda" is the current one
        t = self._on.get(index)
        if t is None:
            if torch.cuda.is_current_stream_capturing():
                raise RuntimeError("a Rotary's first call on a device uploads its frequencies: make it before the capture")
            device = torch.device("cuda", index)
            t = self._on[index] = self._turns.to(device)
            torch.cuda.current_stream(device).synchronize()   # other streams may be the next to read it
        return t

    def __call__(self, q, k, positions, q_out=None, k_out=None, stream=None):
        """Turns q and k (bf16 [T, Hq, D] and [T, Hkv, D], parts of wider rows allowed; either may be None) by
        positions (int32 [T]). Returns (q_out, k_out), by default new tensors; an output may be its input."""
        given = q if q is not None else k
        if given is None:
            return None, None
        t = given.shape[0]
        _dev(positions, "positions", torch.int32, (t,))
        ins = [x for x in (q, k) if x is not None]
        args, outs = [], []
        for x, out, name in ((q, q_out, "q"), (k, k_out, "k")):
            if x is None:
                if out is not None:
                    raise ValueError(f"{name}_out without {name}")
                args += [None, 0, None, 0]
                outs.append(None)
                continue
            if x.dim() != 3:
                raise ValueError(f"{name} must be [tokens, heads, head_dim]")
            shape = (t, x.shape[1], self.head_dim)
            stride = _rows(x, name, shape)
            if out is None:
                with torch.cuda.stream(stream):   # the stream that it is written on
                    out = torch.empty(shape, dtype=torch.bfloat16, device=x.device)
            out_stride = _rows(out, name + "_out", shape)
            _check_turned(x, out, name + "_out", ins)
            args += [x.data_ptr(), stride, out.data_ptr(), out_stride]
            outs.append(out)
        if q_out is not None and k_out is not None and _overlap(q_out, k_out):
            raise ValueError("k_out overlaps q_out")
        device = given.device
        with _on_device(device):
            _check("sf_rotary", lib().sf_rotary(
                self.desc_ref, t, 0 if q is None else q.shape[1], 0 if k is None else k.shape[1],
                self.turns_on(device).data_ptr(), positions.data_ptr(), *args,
                stream.cuda_stream if stream else _current_stream(device)))
        return tuple(outs)


class Sampler:
    """Draws tokens from logits by given uniform numbers, with temperature, top-k, top-p and min-p (sf_sample, whose rules
    these are). Its scratch memory comes from torch's allocator at every call, in the stream's order, so calls on any
    stream may overlap and be captured."""
    DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}

    def __init__(self, device=None):
        self.device = torch.device("cuda" if device is None else device)
        self._L = lib()
        self._last = (None, None, 0)   # (shape, desc, workspace bytes) of the last call

    def __call__(self, logits, uniform, temperature=None, top_k=None, top_p=None, min_p=None, token=None, logprob=None,
                 kept=None, stream=None):
        """logits: fp32, bf16 or fp16 [B, V], rows may lie apart; uniform: fp32 [B] in [0, 1); temperature, top_p,
        min_p: fp32 [B] or None (1, no cut), top_k: int32 [B] or None. Returns (token int32, logprob fp32, kept fp32),
        each [B], into the tensors given."""
        if not isinstance(logits, torch.Tensor) or logits.dim() != 2 or not logits.is_cuda:
            raise ValueError("logits must be a GPU tensor [rows, vocab]")
        code = self.DTYPES.get(logits.dtype)
        if code is None:
            raise ValueError(f"logits must be float32, bfloat16 or float16 (got {logits.dtype})")
        b, v = logits.shape
        if max(b, v) >= 1 << 31:
            raise ValueError(f"logits of {b} x {v} are more than a call takes")
        stride = logits.stride(0) if b > 1 else v
        if (v > 1 and logits.stride(1) != 1) or stride < v:
            raise ValueError("a row's logits must be contiguous, and rows must not overlap")
        _dev(uniform, "uniform", torch.float32, (b,))
        for t, name, dtype in ((temperature, "temperature", torch.float32), (top_k, "top_k", torch.int32),
                               (top_p, "top_p", torch.float32), (min_p, "min_p", torch.float32)):
            if t is not None:
                _dev(t, name, dtype, (b,))
        key = (b, v, stride, code)
        last, desc, size = self._last
        if key != last:   # kept only once it is known to be good
            desc, need = sf_sample_desc(*key, 0), ctypes.c_uint64()
            _check("sf_sample_workspace", self._L.sf_sample_workspace(ctypes.byref(desc), ctypes.byref(need)))
            size = need.value
            self._last = (key, desc, size)
        with _on_device(logits.device), torch.cuda.stream(stream) if stream else _HERE:
            made = []
            for t, name, dtype in ((token, "token", torch.int32), (logprob, "logprob", torch.float32), (kept, "kept", torch.float32)):
                made.append(torch.empty((b,), dtype=dtype, device=logits.device) if t is None else _dev(t, name, dtype, (b,)))
            workspace = torch.empty((max(16, size),), dtype=torch.uint8, device=logits.device)
            _check("sf_sample", self._L.sf_sample(
                ctypes.byref(desc), logits.data_ptr(), _addr(temperature), _addr(top_k), _addr(top_p), _addr(min_p),
                uniform.data_ptr(), made[0].data_ptr(), made[1].data_ptr(), made[2].data_ptr(), workspace.data_ptr(),
                size, stream.cuda_stream if stream else _current_stream(logits.device)))
        return tuple(made)


class PageTable:
    """Host bookkeeping of a growing paged cache: the page pool and a host copy
    of the block table.

    Each decode step generates one token per running trajectory (App. B.1).
    advance(lens) moves to the next step's lengths (0 for a sequence that has
    left) and
      1. returns to the pool every page of the sequences that have left since
         the previous step (ascending sequence order, each in block-table order);
      2. if appending, takes one page for every newest token that opens a page
         (index L - 1 a multiple of 16), in ascending sequence order, and
         records it in the host block table.
    It returns the int32 [B] new-page array the append kernel takes (-1 where
    the token lands in a page the sequence already holds).

    groups = (group_offsets, shared_lens): sequences group_offsets[i] .. group_offsets[i+1] - 1 start with the same
    shared_lens[i] // 16 pages, which are free once the last of them has left.
    """

    def __init__(self, num_pages, bt_host, lens0, groups=None):
        self.bt = np.array(bt_host, dtype=np.int32, order="C", copy=True)
        lens0 = np.asarray(lens0, dtype=np.int64)
        self.pool = PagePool(num_pages)
        npg = (lens0 + PAGE - 1) // PAGE
        common = np.zeros(lens0.size, dtype=np.int64)   # pages whose first holder is an earlier member
        shared = []
        if groups is not None:
            _, offsets, counts = _host_groups(lens0.size, lens0, *groups)
            if offsets[0] != 0 or offsets[-1] != lens0.size or np.any(np.diff(offsets) < 0) or np.any(counts < 0):
                raise ValueError("groups must cover the sequences one behind the other")
            for a, b, tokens in zip(offsets[:-1].tolist(), offsets[1:].tolist(), counts.tolist()):
                live = [s for s in range(a, b) if lens0[s] > 0]
                if any(lens0[s] < tokens for s in live):
                    raise ValueError("a member is shorter than its group's shared tokens")
                for s in live[1:]:
                    common[s] = tokens // PAGE
                    if not np.array_equal(self.bt[s, : common[s]], self.bt[live[0], : common[s]]):
                        raise ValueError("members of a group must start with the same pages")
                    shared.append(self.bt[s, : common[s]])
        held = [self.bt[s, common[s]: npg[s]] for s in range(lens0.size)]
        self.pool.claim(np.concatenate(held) if held else np.zeros(0, np.int32))
        if shared:
            self.pool.share(np.concatenate(shared))
        self.prev = np.ascontiguousarray(lens0, dtype=np.int32)
        self.new_pages = np.empty(lens0.size, dtype=np.int32)

    def advance(self, lens, appending=True) -> np.ndarray:
        """The library's sf_page_table_step on the host table; returns new_pages."""
        lens = np.ascontiguousarray(lens, dtype=np.int32)
        if lens.shape != self.prev.shape:
            raise ValueError("lens must have one entry per sequence")
        _check("sf_page_table_step", self.pool._L.sf_page_table_step(
            self.pool._p, self.bt.ctypes.data, self.bt.shape[1], lens.size, self.prev.ctypes.data,
            lens.ctypes.data, int(bool(appending)), self.new_pages.ctypes.data))
        self.prev = lens
        return self.new_pages


    def truncate(self, keep) -> None:
        """After an eviction: the sequences hold keep tokens, and the pages behind them go back to the pool
        (the library's sf_page_table_truncate on the host table; the next advance continues from keep)."""
        keep = _host_i32(keep, "keep", self.prev.size)
        _check("sf_page_table_truncate", self.pool._L.sf_page_table_truncate(
            self.pool._p, self.bt.ctypes.data, self.bt.shape[1], keep.size, self.prev.ctypes.data, keep.ctypes.data))
        self.prev = keep.copy()


class DecodeLoopRunner:
    """Multi-step decode over a growing paged cache: per step, PageTable
    bookkeeping on the host, then append-then-attend and the merge of split
    sequences on the GPU. The first step (the prompt) only attends.
    block_table is the device table the kernels read and extend. With fp8 =
    (k_scale, v_scale) the pools are an fp8 cache. A loop with a budget calls
    key_weights after its steps and evict every so many of them; the lengths of
    the step after an eviction go on from the kept tokens.

    rotary (a Rotary): q and k_new come as the projections give them, and are turned by their positions
    (the keys of the cache at the start are turned already). groups = (group_offsets, shared_lens): trajectories sampled
    from common prompts, as for DecodeAttention.shared and PageTable; such a loop neither evicts nor weighs keys (a
    page that several sequences hold has no weights of one's own), and a sequence that has left does not
    start again. With either, new tokens are stored before the attention (and over bf16 pools attended to as stored)."""

    def __init__(self, num_q_heads, num_kv_heads, head_dim, k_pool, v_pool, block_table, bt_host, lens0,
                 scale, device=None, num_cus=None, attn=None, fp8=None, rotary=None, groups=None):
        """attn: an existing DecodeAttention of the same head geometry to reuse
        (its native runner keeps its pinned ring and workspace across loops)."""
        if attn is not None and (attn.hq, attn.hkv, attn.d) != (int(num_q_heads), int(num_kv_heads), int(head_dim)):
            raise ValueError("attn was made for another head geometry")
        self.attn = attn or DecodeAttention(num_q_heads, num_kv_heads, head_dim, device=device, num_cus=num_cus)
        self.k_pool, self.v_pool, self.block_table, self.scale = k_pool, v_pool, block_table, float(scale)
        self.table = PageTable(k_pool.shape[0], bt_host, lens0, groups)
        self.fp8, self.rotary = fp8, rotary
        self.groups = None if groups is None else _host_groups(len(lens0), lens0, *groups)[1:]
        self.evicted = np.zeros(self.table.prev.size, dtype=np.int32)   # tokens given up so far, per sequence
        self.weighed = np.zeros_like(self.evicted)   # cached tokens that have weights
        self.steps = 0

    @property
    def bt_host(self):
        return self.table.bt

    @property
    def pool(self):
        return self.table.pool

    def step(self, q, lens, k_new=None, v_new=None, out=None, lse=None, stream=None, attn_events=None):
        lens = np.asarray(lens, dtype=np.int64)
        appending = self.steps > 0
        if appending and (k_new is None or v_new is None):
            raise ValueError("every step after the first appends a token: pass k_new and v_new")
        if self.groups is not None and np.any((lens > 0) & (self.table.prev == 0)):
            raise ValueError("a sequence of a group that has left does not start again")
        if self.groups is not None and attn_events is not None:
            raise ValueError("a step over groups takes no attn_events")
        if self.groups is not None and np.any((lens > 0) & (lens < np.repeat(self.groups[1], np.diff(self.groups[0])))):
            raise ValueError("a member is shorter than its group's shared tokens")
        new_pages = self.table.advance(lens, appending)
        if DEBUG_CHECKS:
            desc = make_desc(lens.size, self.attn.hq, self.attn.hkv, self.attn.d, self.table.bt.shape[1],
                             self.k_pool.shape[0], self.scale)
            check_block_table(desc, self.table.bt, lens)
            self.attn._host_checked = True
        append = (k_new, v_new, new_pages) if appending else None
        if self.rotary is None and self.groups is None:
            out = self.attn(q, self.k_pool, self.v_pool, self.block_table, lens.astype(np.int32), self.scale,
                            out=out, lse=lse, stream=stream, attn_events=attn_events, append=append, fp8=self.fp8)
        else:
            out = self._step_stored(q, lens.astype(np.int32), append, out, lse, stream, attn_events)
        self.steps += 1
        if not lens.all():   # sequences that are not running: one that starts there later has nothing of theirs
            self.evicted, self.weighed = (np.where(lens > 0, x, 0) for x in (self.evicted, self.weighed))
        return out

    def _step_stored(self, q, lens, append, out, lse, stream, attn_events):
        """A step of a loop with rotary positions or groups: what is new is turned and stored, then attended to."""
        attn, checked = self.attn, self.attn._host_checked
        if self.rotary is not None and (append is None or self.fp8 is not None):
            with torch.cuda.stream(stream):
                at = torch.from_numpy(np.maximum(lens - 1 + self.evicted, 0).astype(np.int32)).to(q.device)
                q, k = self.rotary(q, None if append is None else append[0], at, stream=stream)
            if append is not None:
                append = (k, *append[1:])
        if append is not None and self.fp8 is None:
            first = np.maximum(lens - 1 + self.evicted, 0).astype(np.int32)
            turned = attn.rotate_store(self.rotary, q if self.rotary is not None else None, append[0], append[1], self.k_pool,
                                       self.v_pool, self.block_table, lens, first_pos=first, new_pages=append[2], stream=stream)
            q, append = q if turned is None else turned, None
        elif append is not None and self.groups is not None:
            rows = np.flatnonzero(lens > 0)
            k, v = append[0], append[1]
            if rows.size < lens.size:   # the store takes the running sequences' rows
                with torch.cuda.stream(stream):
                    at = torch.from_numpy(rows).to(q.device)
                    k, v = k[at], v[at]
            attn._host_checked = checked
            attn.store_fp8(k, v, self.k_pool, self.v_pool, self.fp8, self.block_table, lens, (lens > 0).astype(np.int32),
                           new_pages=append[2], stream=stream)
            append = None
        attn._host_checked = checked
        if self.groups is None:
            return attn(q, self.k_pool, self.v_pool, self.block_table, lens, self.scale, out=out, lse=lse, stream=stream,
                        attn_events=attn_events, append=append, fp8=self.fp8)
        return attn.shared(q, self.k_pool, self.v_pool, self.block_table, lens, *self.groups, self.scale, out=out, lse=lse,
                           fp8=self.fp8, stream=stream)

    def key_weights(self, q, lse, weights, positions, stream=None):
        """Adds the last step's attention weights (its q and lse, or their rows of the running sequences) to weights.
        Tokens that no call has weighed start there, and get their positions. q as the step took it: with rotary positions
        it is turned here as it was there."""
        if self.groups is not None:
            raise ValueError("a loop over groups weighs no keys")
        lens = self.table.prev
        live = lens > 0
        if not live.all() and q.shape[0] == lse.shape[0] == lens.size:
            if not live.any():
                return
            edges = np.flatnonzero(np.diff(live, prepend=False, append=False)).reshape(-1, 2).tolist()
            with torch.cuda.stream(stream):   # where the rows are read
                q, lse = (torch.cat([x[a:b] for a, b in edges]) for x in (q, lse))
        if self.rotary is not None and live.any():
            with torch.cuda.stream(stream):
                at = torch.from_numpy((lens - 1 + self.evicted)[live].astype(np.int32)).to(q.device)
                q, _ = self.rotary(q, None, at, stream=stream)
        held = np.minimum(self.weighed, lens)
        self.attn.key_weights(q, lse, self.k_pool, self.block_table, lens, (lens > 0).astype(np.int32), self.scale, weights,
                              positions=positions, held_lens=held, first_pos=held + self.evicted,
                              k_scale=None if self.fp8 is None else self.fp8[0], stream=stream)
        self.weighed = lens.copy()

    def evict(self, keep, weights, positions, sinks=0, recent=0, stream=None):
        """Evicts every running sequence to at most keep tokens and frees the pages behind them. Returns the lengths.
        Every cached token must have weights: key_weights comes first."""
        if self.groups is not None:
            raise ValueError("a loop over groups does not evict")
        lens = self.table.prev
        if not np.array_equal(self.weighed, lens):
            raise ValueError("tokens without weights: call key_weights after the last step")
        kept = np.minimum(lens, keep).astype(np.int32)
        self.attn.evict(self.k_pool, self.v_pool, self.block_table, lens, kept, weights, positions,
                        ends=lens + self.evicted, sinks=sinks, recent=recent, fp8=self.fp8, stream=stream)
        self.table.truncate(kept)
        self.evicted = self.evicted + (lens - kept)
        self.weighed = kept.copy()
        return kept
