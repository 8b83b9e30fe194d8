"""Thin ctypes binding of libsplash_attn (include/splash_attn.h).

Argument marshalling only: every step of the attention path runs in the
library's gfx950 kernels.  Tensors are torch tensors on the GPU; their device
pointers and the current HIP stream are handed to the C entry points of the
same names.  A missing library raises: there is no fallback.
"""
from __future__ import annotations

import ctypes
import os
import struct
from typing import Optional

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libsplash_attn.so")

SPLASH_OK = 0
SPLASH_ERR_INVALID_ARGUMENT = -1
SPLASH_ERR_UNSUPPORTED = -2
SPLASH_ERR_MISALIGNED = -3
SPLASH_ERR_WORKSPACE_TOO_SMALL = -4
SPLASH_ERR_HIP = -5

KV_BF16 = 0
KV_FP8_E4M3 = 1
KV_FP8_LATENT = 2   # 656-byte rows: E4M3 latent, 4 fp32 tile scales, bf16 RoPE
FLAG_DEBUG_CHECK = 1
FLAG_FORCE_SPLIT = 2
FLAG_EXACT_QK = 4
DEFAULT_MAX_PARTIALS = 1024
GQA_E4M3 = 0
GQA_INT8 = 1


class SplashError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{message} (status {status})")
        self.status = status


class MlaDesc(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32),
        ("num_heads", ctypes.c_int32),
        ("dim_qk", ctypes.c_int32),
        ("dim_v", ctypes.c_int32),
        ("page_size", ctypes.c_int32),
        ("max_pages_per_seq", ctypes.c_int32),
        ("num_pages", ctypes.c_int32),
        ("kv_dtype", ctypes.c_int32),
        ("kv_scales", ctypes.c_void_p),
        ("softmax_scale", ctypes.c_float),
        ("flags", ctypes.c_uint32),
        ("split_pages", ctypes.c_int32),
    ]


class GqaDesc(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32),
        ("num_heads", ctypes.c_int32),
        ("num_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("page_size", ctypes.c_int32),
        ("max_pages_per_seq", ctypes.c_int32),
        ("num_pages", ctypes.c_int32),
        ("code_type", ctypes.c_int32),
        ("softmax_scale", ctypes.c_float),
    ]


class RopeView(ctypes.Structure):
    _fields_ = [
        ("x", ctypes.c_void_p),
        ("y", ctypes.c_void_p),
        ("x_token_stride", ctypes.c_int64),
        ("x_head_stride", ctypes.c_int64),
        ("y_token_stride", ctypes.c_int64),
        ("y_head_stride", ctypes.c_int64),
        ("num_heads", ctypes.c_int32),
    ]


class RopeDesc(ctypes.Structure):
    _fields_ = [
        ("rot_dim", ctypes.c_int32),
        ("interleaved", ctypes.c_int32),
        ("num_axes", ctypes.c_int32),
        ("scale", ctypes.c_float),
        ("inv_freq", ctypes.POINTER(ctypes.c_double)),
        ("pair_axis", ctypes.POINTER(ctypes.c_uint8)),
    ]


_lib = None

_VP = ctypes.c_void_p
_I32 = ctypes.c_int32
_SZ = ctypes.c_size_t
_PD = ctypes.POINTER(MlaDesc)
_PI32 = ctypes.POINTER(ctypes.c_int32)
_I64 = ctypes.c_int64
_PG = ctypes.POINTER(GqaDesc)

_SIGNATURES = {
    "splash_mla_workspace_size": (_SZ, [_I32, _I32, _I32, _I32]),
    "splash_mla_workspace_offsets": (_SZ, [_I32, _I32, _I32, _I32, ctypes.POINTER(_SZ)]),
    "splash_mla_attend": (ctypes.c_int, [_VP, _VP, _VP, _VP, _I32, _VP, _VP, _PD, _VP, _SZ, _VP]),
    "splash_mla_attend_noalloc": (ctypes.c_int, [_VP, _VP, _VP, _VP, _I32, _VP, _VP, _PD, _VP]),
    "splash_mla_plan": (ctypes.c_int, [_VP, _I32, _PD, _VP, _SZ, _VP]),
    "splash_mla_run": (ctypes.c_int, [_VP, _VP, _VP, _VP, _I32, _VP, _VP, _PD, _VP, _SZ, _VP]),
    "splash_mla_attend_units": (ctypes.c_int, [_VP, _VP, _VP, _VP, _I32, _VP, _VP, _PD, _VP, _SZ, _VP]),
    "splash_mla_combine_splits": (ctypes.c_int, [_I32, _VP, _VP, _PD, _VP, _SZ, _VP]),
    "splash_mla_combine": (ctypes.c_int, [_VP, _VP, _VP, _I32, _I32, _I32, _VP, _VP, _VP]),
    "splash_mla_attend_topk": (ctypes.c_int, [_VP, _VP, _VP, _VP, _I32, _VP, _VP, _I32, _VP, _VP, _PD, _VP, _SZ,
                                              _VP]),
    "splash_dop_pack_q": (ctypes.c_int, [_VP, _VP, _VP, _I32, _I32, _VP, _VP]),
    "splash_dop_unpack_q": (ctypes.c_int, [_VP, _I32, _I32, _I32, _VP, _VP]),
    "splash_dop_pack_out": (ctypes.c_int, [_VP, _I32, _I32, _I32, _VP, _VP]),
    "splash_dop_unpack_out": (ctypes.c_int, [_VP, _VP, _I32, _I32, _VP, _VP]),
    "splash_mla_attend_shard": (ctypes.c_int, [_VP, _VP, _VP, _VP, _I32, _VP, _VP, _I32, _I32, _VP, _VP, _PD, _VP,
                                               _SZ, _VP]),
    "splash_mla_debug_gather": (ctypes.c_int, [_VP, _VP, _VP, _PD, _VP, _VP]),
    "splash_mla_plan_host": (ctypes.c_int, [_PI32, _I32, _PD, _I32, _I32, _PI32, _I32, _PI32, _PI32, _PI32]),
    "splash_mla_max_units": (_I32, [_I32, _I32, _I32]),
    "splash_device_workers": (_I32, []),
    "splash_step_tables": (ctypes.c_int, [_VP, _VP, _I32, _I32, _VP, _I32, _VP, _VP, _VP, _I32, _I32, _I32, _VP, _VP, _VP,
                                          _VP, _VP]),
    "splash_rope": (ctypes.c_int, [_VP, _I32, _VP, _I64, _I32, ctypes.POINTER(RopeDesc), _VP]),
    "splash_gqa_append": (ctypes.c_int, [_VP, _VP, _I64, _I64, _VP, _I32, _VP, _VP, _VP, _VP, _PG, _VP]),
    "splash_gqa_workspace_size": (_SZ, [_PG, _I32]),
    "splash_gqa_attend": (ctypes.c_int, [_VP, _VP, _VP, _VP, _VP, _VP, _VP, _I32, _VP, _VP, _PG, _VP, _SZ, _VP]),
    "splash_status_string": (ctypes.c_char_p, [ctypes.c_int]),
    "splash_last_error": (ctypes.c_char_p, []),
    "splash_version": (ctypes.c_char_p, []),
}


def _hip_runtimes_mapped():
    try:
        with open("/proc/self/maps") as f:
            return sorted({l.split()[-1] for l in f if "libamdhip64" in l})
    except OSError:
        return []


def lib():
    """Load libsplash_attn.so (built in-tree); raise if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2609_37626_amd.build`")
    import torch  # noqa: F401  (load torch's HIP runtime first so the library binds to it)
    handle = ctypes.CDLL(LIB_PATH)
    for name, (res, args) in _SIGNATURES.items():
        fn = getattr(handle, name)
        fn.restype = res
        fn.argtypes = args
    runtimes = _hip_runtimes_mapped()
    if len(runtimes) > 1:
        raise RuntimeError(f"two HIP runtimes are mapped into this process: {runtimes}")
    _lib = handle
    return _lib


def _check(status: int) -> None:
    if status != SPLASH_OK:
        L = lib()
        raise SplashError(status, f"{L.splash_status_string(status).decode()}: {L.splash_last_error().decode()}")


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream(stream) -> Optional[int]:
    if stream is not None:
        return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)
    return _current_stream()


def _current_stream() -> int:
    """The current HIP stream of the current device, as the C side takes it.
    (Once the device is initialised, straight from the runtime binding, where
    this torch has it: building a torch Stream object for its handle was a
    third of the 7.4 us that a regroup call spent on the host.)"""
    import torch
    if torch.cuda.is_initialized():
        try:
            return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
        except AttributeError:
            pass
    return torch.cuda.current_stream().cuda_stream


def make_desc(batch: int, num_heads: int, max_pages_per_seq: int, num_pages: int,
              kv_dtype: int = KV_BF16, kv_scales=None, softmax_scale: float = 1.0 / 192 ** 0.5,
              flags: int = 0, split_pages: int = 0) -> MlaDesc:
    d = MlaDesc()
    d.batch = batch
    d.num_heads = num_heads
    d.dim_qk = 576
    d.dim_v = 512
    d.page_size = 64
    d.max_pages_per_seq = max_pages_per_seq
    d.num_pages = num_pages
    d.kv_dtype = kv_dtype
    d.kv_scales = _ptr(kv_scales)
    d.softmax_scale = float(np.float32(softmax_scale))
    d.flags = flags
    d.split_pages = split_pages
    return d


def workspace_size(batch: int, q_chunk: int, num_heads: int, max_partials: int = 0) -> int:
    return int(lib().splash_mla_workspace_size(batch, q_chunk, num_heads, max_partials))


def workspace_offsets(batch: int, q_chunk: int, num_heads: int, max_partials: int = 0):
    offs = (_SZ * 6)()
    total = lib().splash_mla_workspace_offsets(batch, q_chunk, num_heads, max_partials, offs)
    return list(offs), int(total)


def device_workers() -> int:
    return int(lib().splash_device_workers())


def splash_mla_attend(q, kv_pages, block_table, seq_lens, q_chunk: int, out, lse, desc: MlaDesc,
                      workspace, stream=None) -> None:
    _check(lib().splash_mla_attend(_ptr(q), _ptr(kv_pages), _ptr(block_table), _ptr(seq_lens), q_chunk,
                                   _ptr(out), _ptr(lse), ctypes.byref(desc), _ptr(workspace),
                                   workspace.numel() * workspace.element_size(), _stream(stream)))


def splash_mla_attend_noalloc(q, kv_pages, block_table, seq_lens, q_chunk: int, out, lse, desc: MlaDesc,
                              stream=None) -> None:
    """splash_mla_attend on the library's own workspace (no allocation)."""
    _check(lib().splash_mla_attend_noalloc(_ptr(q), _ptr(kv_pages), _ptr(block_table), _ptr(seq_lens), q_chunk,
                                           _ptr(out), _ptr(lse), ctypes.byref(desc), _stream(stream)))


NOALLOC_SCRATCH_BYTES = 128 << 20  # SPLASH_NOALLOC_SCRATCH_BYTES


def splash_mla_plan(seq_lens, q_chunk: int, desc: MlaDesc, workspace, stream=None) -> None:
    _check(lib().splash_mla_plan(_ptr(seq_lens), q_chunk, ctypes.byref(desc), _ptr(workspace),
                                 workspace.numel() * workspace.element_size(), _stream(stream)))


def splash_mla_run(q, kv_pages, block_table, seq_lens, q_chunk: int, out, lse, desc: MlaDesc,
                   workspace, stream=None) -> None:
    _check(lib().splash_mla_run(_ptr(q), _ptr(kv_pages), _ptr(block_table), _ptr(seq_lens), q_chunk,
                                _ptr(out), _ptr(lse), ctypes.byref(desc), _ptr(workspace),
                                workspace.numel() * workspace.element_size(), _stream(stream)))


def splash_mla_attend_units(q, kv_pages, block_table, seq_lens, q_chunk: int, out, lse, desc: MlaDesc,
                            workspace, stream=None) -> None:
    _check(lib().splash_mla_attend_units(_ptr(q), _ptr(kv_pages), _ptr(block_table), _ptr(seq_lens), q_chunk,
                                         _ptr(out), _ptr(lse), ctypes.byref(desc), _ptr(workspace),
                                         workspace.numel() * workspace.element_size(), _stream(stream)))


def splash_mla_combine_splits(q_chunk: int, out, lse, desc: MlaDesc, workspace, stream=None) -> None:
    _check(lib().splash_mla_combine_splits(q_chunk, _ptr(out), _ptr(lse), ctypes.byref(desc), _ptr(workspace),
                                           workspace.numel() * workspace.element_size(), _stream(stream)))


def splash_mla_attend_shard(q, kv_pages, block_table, seq_lens, q_chunk: int, key_begin, key_end,
                            num_shards: int, shard: int, part_out, part_lse, desc: MlaDesc, workspace,
                            stream=None) -> None:
    _check(lib().splash_mla_attend_shard(_ptr(q), _ptr(kv_pages), _ptr(block_table), _ptr(seq_lens), q_chunk,
                                         _ptr(key_begin), _ptr(key_end), num_shards, shard, _ptr(part_out),
                                         _ptr(part_lse), ctypes.byref(desc), _ptr(workspace),
                                         workspace.numel() * workspace.element_size(), _stream(stream)))


def splash_mla_attend_topk(q, kv_pages, block_table, seq_lens, q_chunk: int, topk_idx, topk_count, out, lse,
                           desc: MlaDesc, workspace, stream=None) -> None:
    """Row n attends the positions topk_idx[n, :topk_count[n]] of its request's history."""
    _check(lib().splash_mla_attend_topk(_ptr(q), _ptr(kv_pages), _ptr(block_table), _ptr(seq_lens), q_chunk,
                                        _ptr(topk_idx), _ptr(topk_count), int(topk_idx.shape[1]), _ptr(out), _ptr(lse),
                                        ctypes.byref(desc), _ptr(workspace),
                                        workspace.numel() * workspace.element_size(), _stream(stream)))


def splash_dop_pack_q(q_nope, q_rope, row_order, send, stream=None) -> None:
    """Rank side: send[k] = q_nope[row_order[k]] | q_rope[row_order[k]] (all local heads)."""
    n, hl = q_nope.shape[:2]
    _check(lib().splash_dop_pack_q(_ptr(q_nope), _ptr(q_rope), _ptr(row_order), n, hl, _ptr(send), _stream(stream)))


def splash_dop_unpack_q(recv, num_ranks: int, q_owner, stream=None) -> None:
    """Owner side: recv [T, n, H/T, 576] -> q_owner [n, H, 576]."""
    n, H = q_owner.shape[:2]
    _check(lib().splash_dop_unpack_q(_ptr(recv), num_ranks, n, H // num_ranks, _ptr(q_owner), _stream(stream)))


def splash_dop_pack_out(out_owner, num_ranks: int, send, stream=None) -> None:
    """Owner side: out_owner [n, H, 512] -> send [T, n, H/T, 512]."""
    n, H = out_owner.shape[:2]
    _check(lib().splash_dop_pack_out(_ptr(out_owner), num_ranks, n, H // num_ranks, _ptr(send), _stream(stream)))


def splash_dop_unpack_out(recv, row_order, out, stream=None) -> None:
    """Rank side: out[row_order[k]] = recv[k] (all local heads)."""
    n, hl = out.shape[:2]
    _check(lib().splash_dop_unpack_out(_ptr(recv), _ptr(row_order), n, hl, _ptr(out), _stream(stream)))


def splash_mla_combine(partials, partial_lse, split_indptr, batch: int, q_chunk: int, num_heads: int,
                       out, out_lse=None, stream=None) -> None:
    _check(lib().splash_mla_combine(_ptr(partials), _ptr(partial_lse), _ptr(split_indptr), batch, q_chunk,
                                    num_heads, _ptr(out), _ptr(out_lse), _stream(stream)))


def splash_mla_debug_gather(kv_pages, block_table, seq_lens, desc: MlaDesc, dense_out, stream=None) -> None:
    _check(lib().splash_mla_debug_gather(_ptr(kv_pages), _ptr(block_table), _ptr(seq_lens), ctypes.byref(desc),
                                         _ptr(dense_out), _stream(stream)))


def splash_mla_plan_host(seq_lens: np.ndarray, q_chunk: int, desc: MlaDesc, num_workers: int,
                         max_partials: int = 0):
    """Host mirror of the planner: returns (units [U,4], indptr [T+1], stats dict).

    stats["fold"] tells a fold plan (each worker runs its own units) from a
    plan of one unit size (workers draw units from a queue); for a fold plan
    stats["cap"] is the pages a long tile keeps and stats["worker_start"]
    the first unit of each of the num_workers workers and the end
    (num_workers + 1 entries), else None.
    """
    L = lib()
    seq = np.ascontiguousarray(seq_lens, dtype=np.int32)
    T = int(seq.shape[0]) * q_chunk
    max_units = int(L.splash_mla_max_units(int(seq.shape[0]), q_chunk, max_partials))
    units = np.zeros((max(max_units, 1), 4), dtype=np.int32)
    indptr = np.zeros(T + 1, dtype=np.int32)
    stats = np.zeros(7, dtype=np.int32)
    wstart = np.zeros(num_workers + 1, dtype=np.int32)
    as_p = lambda a: a.ctypes.data_as(_PI32)
    _check(L.splash_mla_plan_host(as_p(seq), q_chunk, ctypes.byref(desc), num_workers, max_partials,
                                  as_p(units), max_units, as_p(indptr), as_p(stats), as_p(wstart)))
    n = int(stats[0])
    fold = int(stats[4]) > 0
    return units[:n].copy(), indptr, {"units": n, "partials": int(stats[1]), "chunk_pages": int(stats[2]),
                                      "total_pages": int(stats[3]), "fold": fold, "cap": int(stats[5]),
                                      "max_parts": int(stats[6]), "worker_start": wstart if fold else None}


# ------------------------------ the serving step around grouped-query attention
#
# These calls check their tensors against what the kernels assume (type, shape,
# strides, one device), run on the tensors' device, and take its current stream.

def _refuse(message: str):
    raise SplashError(SPLASH_ERR_INVALID_ARGUMENT, message)


_I32T = _F32T = _BF16T = None  # torch's types, and the calls that name the device and its current stream (set by _types)
_device = _raw_stream = None
_CODES = {}  # code_type: the types of its pages


def _types():
    global _I32T, _F32T, _BF16T, _device, _raw_stream
    import torch
    _I32T, _F32T, _BF16T = torch.int32, torch.float32, torch.bfloat16
    _CODES.update({GQA_E4M3: (torch.uint8, torch.float8_e4m3fn), GQA_INT8: (torch.int8,)})
    _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", lambda dev: _current_stream())
    _device = torch._C._cuda_getDevice  # (the calls look at this one: last, for their first use from several threads)


def _refuse_tensors(dev: int, **tensors):
    """Says which tensor is not of its type and shape, contiguous and on the device (name=(tensor, types, shape); a
    shape of None is any).  The calls find that one is by one condition over all of them, in about 2 us."""
    if dev < 0:
        _refuse("tensors must be on the GPU")
    for name, (t, dtypes, shape) in tensors.items():
        if t is None:
            continue
        if t.dtype not in dtypes:
            _refuse(f"{name} must be {' or '.join(str(d) for d in dtypes)} (got {t.dtype})")
        if shape is not None and tuple(t.shape) != tuple(shape):
            _refuse(f"{name} must have shape {tuple(shape)} (got {tuple(t.shape)})")
        if not t.is_contiguous():
            _refuse(f"{name} must be contiguous")
        if t.get_device() != dev:
            _refuse(f"{name} is on another device")
    _refuse("tensors do not match")


def _on_device(dev: int, fn, args, stream) -> None:
    """fn(*args, stream handle) with `dev` current."""
    if _device() == dev:
        status = fn(*args, _raw_stream(dev) if stream is None else _stream(stream))
    else:
        import torch
        with torch.cuda.device(dev):
            status = fn(*args, _stream(stream))
    if status != SPLASH_OK:
        _check(status)


def make_gqa_desc(batch: int, num_heads: int, num_kv_heads: int, head_dim: int, max_pages_per_seq: int, num_pages: int,
                  code_type: int = GQA_E4M3, softmax_scale: Optional[float] = None) -> GqaDesc:
    """softmax_scale: 1 / sqrt(head_dim) by default."""
    d = GqaDesc()
    d.batch = batch
    d.num_heads = num_heads
    d.num_kv_heads = num_kv_heads
    d.head_dim = head_dim
    d.page_size = 64
    d.max_pages_per_seq = max_pages_per_seq
    d.num_pages = num_pages
    d.code_type = code_type
    d.softmax_scale = float(np.float32(head_dim ** -0.5 if softmax_scale is None else softmax_scale))
    return d


def gqa_workspace_size(desc: GqaDesc, q_chunk: int) -> int:
    n = int(lib().splash_gqa_workspace_size(ctypes.byref(desc), q_chunk))
    if n == 0:
        _refuse(lib().splash_last_error().decode())
    return n


def make_rope(rot_dim: int, inv_freq, pair_axis=None, num_axes: Optional[int] = None, interleaved: bool = False,
              scale: float = 1.0) -> RopeDesc:
    """inv_freq: radians per position of each of the rot_dim / 2 pairs; pair_axis: the position axis of each (0)."""
    freq = np.ascontiguousarray(inv_freq, dtype=np.float64)
    if freq.shape != (rot_dim // 2,):
        _refuse(f"inv_freq must hold {rot_dim // 2} frequencies")
    d = RopeDesc()
    d.rot_dim = rot_dim
    d.interleaved = int(bool(interleaved))
    d.scale = scale
    d.inv_freq = freq.ctypes.data_as(ctypes.POINTER(ctypes.c_double))
    d.num_axes = 1
    d.arrays = [freq]  # (kept alive with the descriptor)
    if pair_axis is not None:
        axis = np.asarray(pair_axis, dtype=np.int64)
        if axis.shape != freq.shape or axis.min() < 0 or axis.max() > 3:
            _refuse("pair_axis must hold an axis, 0 to 3, for every pair")
        d.num_axes = int(axis.max()) + 1
        axis = axis.astype(np.uint8)
        d.pair_axis = axis.ctypes.data_as(ctypes.POINTER(ctypes.c_uint8))
        d.arrays.append(axis)
    if num_axes is not None:
        d.num_axes = num_axes
    return d


def splash_step_tables(seq_lens, q_chunk: int, free_pages, taken_in, taken_out, block_table, num_pages: int, new_indptr,
                       slots, positions, requests, new_lens=None, stream=None) -> None:
    """Pages, slots and positions of the step's new tokens (new_lens[b], or q_chunk of every request)."""
    if _device is None:
        _types()
    i32 = _I32T
    b, rows, width, dev = seq_lens.numel(), slots.numel(), block_table.shape[-1], seq_lens.get_device()
    new = seq_lens if new_lens is None else new_lens
    if not (seq_lens.dtype is i32 and new.dtype is i32 and free_pages.dtype is i32 and taken_in.dtype is i32
            and taken_out.dtype is i32 and block_table.dtype is i32 and new_indptr.dtype is i32 and slots.dtype is i32
            and positions.dtype is i32 and requests.dtype is i32
            and new.numel() == b and taken_in.numel() == 2 and taken_out.numel() == 2 and block_table.shape == (b, width)
            and new_indptr.numel() == b + 1 and positions.numel() == rows and requests.numel() == rows
            and seq_lens.is_contiguous() and new.is_contiguous() and free_pages.is_contiguous() and taken_in.is_contiguous()
            and taken_out.is_contiguous() and block_table.is_contiguous() and new_indptr.is_contiguous()
            and slots.is_contiguous() and positions.is_contiguous() and requests.is_contiguous()
            and 0 <= dev == new.get_device() == free_pages.get_device() == taken_in.get_device() == taken_out.get_device()
            == block_table.get_device() == new_indptr.get_device() == slots.get_device() == positions.get_device()
            == requests.get_device()):
        t = (i32,)
        _refuse_tensors(dev, seq_lens=(seq_lens, t, (b,)), new_lens=(new_lens, t, (b,)), free_pages=(free_pages, t, None),
                        taken_in=(taken_in, t, (2,)), taken_out=(taken_out, t, (2,)), block_table=(block_table, t, (b, width)),
                        new_indptr=(new_indptr, t, (b + 1,)), slots=(slots, t, (rows,)), positions=(positions, t, (rows,)),
                        requests=(requests, t, (rows,)))
    _on_device(dev, lib().splash_step_tables, (
        seq_lens.data_ptr(), None if new_lens is None else new.data_ptr(), q_chunk, b, free_pages.data_ptr(),
        free_pages.numel(), taken_in.data_ptr(), taken_out.data_ptr(), block_table.data_ptr(), width, num_pages, rows,
        new_indptr.data_ptr(), slots.data_ptr(), positions.data_ptr(), requests.data_ptr()), stream)


# Two splash_rope_view (a ctypes array takes 1 us longer to fill).
_pack_views = struct.Struct("@PPqqqqi4xPPqqqqi4x").pack
_NO_VIEW = (0,) * 7


def _rope_view(x, y, tokens: int, rot_dim: int, dev: int) -> tuple:
    shape = x.shape
    xs, ys = x.stride(), y.stride()
    if not (x.dtype is _BF16T and y.dtype is _BF16T and x.get_device() == dev == y.get_device() and len(shape) == 3
            and shape == y.shape and shape[0] == tokens and shape[2] == rot_dim and xs[2] == 1 == ys[2]):
        _refuse(f"x and out must be bf16 [{tokens}, heads, {rot_dim}] on the positions' device, the last dimension dense "
                f"(got {x.dtype}, {y.dtype}, {tuple(shape)}, {tuple(y.shape)}, strides {xs}, {ys})")
    return x.data_ptr(), y.data_ptr(), xs[0], xs[1], ys[0], ys[1], shape[1]


def splash_rope(x, positions, rope: RopeDesc, out=None, x2=None, out2=None, stream=None) -> None:
    """Turns x (and x2) [tokens, heads, rot_dim], views of any token and head stride, by positions [tokens] or
    [axes, tokens] (or [tokens] expanded to it) into out (None: in place)."""
    if _device is None:
        _types()
    shape, strides, dev = positions.shape, positions.stride(), positions.get_device()
    axes, n = (1, shape[0]) if len(shape) == 1 else shape if len(shape) == 2 else (0, 0)
    if axes != rope.num_axes or positions.dtype is not _I32T or (n > 1 and strides[-1] != 1) or dev < 0:
        _refuse(f"positions must be int32 [{rope.num_axes}, tokens] on the GPU, dense along the tokens")
    rot = rope.rot_dim
    views = _pack_views(*_rope_view(x, x if out is None else out, n, rot, dev),
                        *(_NO_VIEW if x2 is None else _rope_view(x2, x2 if out2 is None else out2, n, rot, dev)))
    _on_device(dev, lib().splash_rope, (views, 1 if x2 is None else 2, positions.data_ptr(), strides[0] if axes > 1 else n,
                                        n, rope), stream)


def _gqa_cache_ok(desc: GqaDesc, dev: int, k_pages, v_pages, k_scales, v_scales) -> bool:
    scales, code = (desc.num_pages, desc.num_kv_heads), k_pages.dtype
    pool = (*scales, 64, desc.head_dim)
    return (k_pages.shape == pool and v_pages.shape == pool and k_scales.shape == scales and v_scales.shape == scales
            and code is v_pages.dtype and code in _CODES.get(desc.code_type, ()) and k_scales.dtype is _F32T and v_scales.dtype is _F32T
            and k_pages.is_contiguous() and v_pages.is_contiguous() and k_scales.is_contiguous() and v_scales.is_contiguous()
            and 0 <= dev == k_pages.get_device() == v_pages.get_device() == k_scales.get_device() == v_scales.get_device())


def _refuse_gqa(desc: GqaDesc, dev: int, k_pages, v_pages, k_scales, v_scales, **tensors):
    scales, codes = (desc.num_pages, desc.num_kv_heads), _CODES.get(desc.code_type, ())
    if not codes:
        _refuse(f"unknown code_type {desc.code_type}")
    pool = scales + (64, desc.head_dim)
    _refuse_tensors(dev, k_pages=(k_pages, codes, pool), v_pages=(v_pages, codes, pool),
                    k_scales=(k_scales, (_F32T,), scales), v_scales=(v_scales, (_F32T,), scales), **tensors)


def splash_gqa_append(k_new, v_new, slots, k_pages, v_pages, k_scales, v_scales, desc: GqaDesc, stream=None) -> None:
    """Row t of k_new and v_new [rows, kv heads, head_dim] (views of one token and head stride) to slot slots[t]."""
    if _device is None:
        _types()
    n, dev = slots.numel(), slots.get_device()
    shape, strides = (n, desc.num_kv_heads, desc.head_dim), k_new.stride()
    if not (_gqa_cache_ok(desc, dev, k_pages, v_pages, k_scales, v_scales)
            and slots.dtype is _I32T and slots.is_contiguous() and k_new.dtype is _BF16T and v_new.dtype is _BF16T
            and k_new.shape == shape and v_new.shape == shape and dev == k_new.get_device() == v_new.get_device()
            and strides == v_new.stride() and strides[2] == 1):
        if k_new.shape == shape and v_new.shape == shape and (strides != v_new.stride() or strides[2] != 1):
            _refuse("k_new and v_new must have the same strides, the last dimension dense")
        bf16 = (_BF16T,)
        _refuse_gqa(desc, dev, k_pages, v_pages, k_scales, v_scales, slots=(slots, (_I32T,), (n,)),
                    k_new=(k_new.contiguous(), bf16, shape), v_new=(v_new.contiguous(), bf16, shape))
    _on_device(dev, lib().splash_gqa_append, (
        k_new.data_ptr(), v_new.data_ptr(), strides[0], strides[1], slots.data_ptr(), n, k_pages.data_ptr(),
        v_pages.data_ptr(), k_scales.data_ptr(), v_scales.data_ptr(), desc), stream)


def splash_gqa_attend(q, k_pages, v_pages, k_scales, v_scales, block_table, seq_lens, q_chunk: int, out, lse,
                      desc: GqaDesc, workspace, stream=None) -> None:
    """lse may be None."""
    if _device is None:
        _types()
    dev, b, heads = q.get_device(), desc.batch, desc.num_heads
    rows, table = (b * q_chunk, heads, desc.head_dim), (b, desc.max_pages_per_seq)
    if not (_gqa_cache_ok(desc, dev, k_pages, v_pages, k_scales, v_scales)
            and q.dtype is _BF16T and out.dtype is _BF16T and q.shape == rows and out.shape == rows
            and block_table.dtype is _I32T and block_table.shape == table and seq_lens.dtype is _I32T
            and seq_lens.numel() == b and workspace.element_size() == 1
            and (lse is None or (lse.dtype is _F32T and lse.shape == rows[:2] and lse.is_contiguous() and lse.get_device() == dev))
            and q.is_contiguous() and out.is_contiguous() and block_table.is_contiguous() and seq_lens.is_contiguous()
            and workspace.is_contiguous() and dev == out.get_device() == block_table.get_device() == seq_lens.get_device()
            == workspace.get_device()):
        import torch
        bf16, i32 = (_BF16T,), (_I32T,)
        _refuse_gqa(desc, dev, k_pages, v_pages, k_scales, v_scales, q=(q, bf16, rows), out=(out, bf16, rows),
                    lse=(lse, (_F32T,), rows[:2]), block_table=(block_table, i32, table), seq_lens=(seq_lens, i32, (b,)),
                    workspace=(workspace, (torch.uint8, torch.int8), None))
    _on_device(dev, lib().splash_gqa_attend, (
        q.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(), k_scales.data_ptr(), v_scales.data_ptr(),
        block_table.data_ptr(), seq_lens.data_ptr(), q_chunk, out.data_ptr(), None if lse is None else lse.data_ptr(), desc,
        workspace.data_ptr(), workspace.numel()), stream)


def version() -> str:
    return lib().splash_version().decode()
