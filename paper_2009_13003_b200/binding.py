"""Thin ctypes binding of ``liblc.so`` (the C ABI in ``include/lc.h``).

Argument marshalling only: every step of the compress and recovery passes runs in the CUDA kernels.
PyTorch supplies device memory (tensors) and the current CUDA stream. There is no CPU fallback: if the
library cannot be loaded the import of this module's functions fails loudly.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
import threading
from typing import NamedTuple

import torch

from . import build as _build

OK, ERR_ARG, ERR_CAPACITY, ERR_NONFINITE, ERR_FORMAT, ERR_MISMATCH, ERR_TIMEOUT, ERR_CUDA, ERR_RANGE, ERR_INDEX = 0, -1, -2, -3, -4, -5, -6, -7, -8, -9
MAX_CHAIN = 8
WAIT_PAGE_BYTES = 128

SYMBOLS = (
    "lc_version", "lc_strerror", "lc_stream_bound", "lc_workspace_bytes", "lc_compress", "lc_compress_update", "lc_compress_timed",
    "lc_recover", "lc_compress_opt", "lc_compress_cached",
    "lc_segments_layout", "lc_compress_segments", "lc_recover_segments", "lc_debug_compress_wait", "lc_debug_update_wait", "lc_merge", "lc_compress_async", "lc_shard_stats", "lc_shard_encode",
    "lc_stream_info", "lc_last_status", "lc_wait", "lc_host_arena_bytes", "lc_compress_host", "lc_recover_host",
    "lc_debug_bins", "lc_debug_codes", "lc_debug_split_segments", "lc_debug_decode_warps",
    "lc_compress_noalloc",
    "lc_q4_bytes", "lc_q4_quantize", "lc_recover_q4", "lc_q4_read", "lc_q4_matvec", "lc_debug_q4_plan",
    "lc_cache_code_bytes", "lc_cache_scale_bytes", "lc_cache_write", "lc_cache_read", "lc_cache_read_pages",
)
NOALLOC_MAX_N = 4194304


class LCInfo(C.Structure):
    _fields_ = [
        ("n", C.c_uint64), ("total_bytes", C.c_uint64), ("payload_bits", C.c_uint64),
        ("payload_offset", C.c_uint64), ("nbits", C.c_uint32), ("nsym", C.c_uint32),
        ("max_len", C.c_uint32), ("nchunks", C.c_uint32), ("valid", C.c_int32), ("fixed_width", C.c_uint32), ("shard", C.c_uint32),
        ("cached_lengths", C.c_uint32), ("mean_rep", C.c_uint32),
    ]


class LCCache(C.Structure):
    _fields_ = [("codes", C.c_void_p), ("scales", C.c_void_p), ("slots", C.c_uint64), ("planes", C.c_uint32), ("heads", C.c_uint32),
                ("dim", C.c_uint32), ("bits", C.c_uint32), ("group", C.c_uint32)]


class LCRows(C.Structure):
    _fields_ = [("data", C.c_void_p), ("row_stride", C.c_uint64), ("head_stride", C.c_uint64)]


class LCError(RuntimeError):
    def __init__(self, code, what=""):
        self.code = code
        super().__init__("%s: %s (%d)" % (what, lib().lc_strerror(code).decode(), code))


_lib = None


def lib():
    """Loads (building first if the shared object is missing or stale and nvcc is present) liblc.so."""
    global _lib
    if _lib is not None:
        return _lib
    path = _build.LIB
    try:
        path = _build.build()
    except Exception as e:  # no nvcc here: use what is in the tree
        if not os.path.exists(path):
            raise RuntimeError("liblc.so is missing and could not be built: %s" % e)
    L = C.CDLL(path)
    u64, i32, vp = C.c_uint64, C.c_int, C.c_void_p
    L.lc_version.restype = i32
    L.lc_strerror.argtypes = [i32]
    L.lc_strerror.restype = C.c_char_p
    L.lc_stream_bound.argtypes = [u64, i32]
    L.lc_stream_bound.restype = u64
    L.lc_workspace_bytes.argtypes = [u64]
    L.lc_workspace_bytes.restype = u64
    L.lc_compress.argtypes = [vp, vp, u64, i32, vp, u64, vp, u64, vp]
    L.lc_compress_update.argtypes = [vp, vp, u64, i32, vp, u64, vp, vp, u64, vp]
    L.lc_compress_opt.argtypes = [vp, vp, u64, i32, vp, u64, vp, vp, u64, C.c_uint32, vp]
    L.lc_compress_cached.argtypes = [vp, vp, u64, i32, vp, u64, vp, vp, u64, vp, vp]
    L.lc_segments_layout.argtypes = [C.POINTER(u64), i32, i32, C.POINTER(u64)]
    L.lc_segments_layout.restype = u64
    L.lc_compress_segments.argtypes = [vp, vp, C.POINTER(u64), i32, i32, vp, u64, vp, vp, u64, vp]
    L.lc_recover_segments.argtypes = [vp, C.POINTER(vp), i32, C.POINTER(u64), i32, i32, vp, vp, u64, vp]
    L.lc_debug_compress_wait.argtypes = [vp, vp, u64, i32, vp, u64, vp, u64, C.c_uint32, C.c_uint32, vp]
    L.lc_debug_update_wait.argtypes = [vp, vp, u64, i32, vp, u64, vp, vp, u64, C.c_uint32, C.c_uint32, vp]
    L.lc_compress_timed.argtypes = [vp, vp, u64, i32, vp, u64, vp, u64, vp, C.POINTER(C.c_float)]
    L.lc_recover.argtypes = [vp, C.POINTER(vp), C.POINTER(u64), i32, u64, vp, vp, u64, vp]
    L.lc_compress_async.argtypes = [vp, vp, u64, i32, vp, u64, vp, u64, vp, vp, vp]
    L.lc_shard_stats.argtypes = [vp, vp, u64, vp, vp, u64, vp]
    L.lc_shard_encode.argtypes = [vp, vp, u64, i32, vp, vp, u64, vp, u64, vp]
    L.lc_merge.argtypes = [vp, C.POINTER(vp), C.POINTER(u64), i32, u64, i32, vp, u64, vp, vp, u64, vp]
    L.lc_stream_info.argtypes = [vp, C.POINTER(LCInfo), vp]
    L.lc_last_status.argtypes = [vp, vp]
    L.lc_wait.argtypes = [vp, vp, C.POINTER(LCInfo), vp, vp]
    L.lc_host_arena_bytes.argtypes = [u64, i32, i32]
    L.lc_host_arena_bytes.restype = u64
    L.lc_compress_host.argtypes = [vp, vp, u64, i32, vp, u64, C.POINTER(u64), vp, u64, vp]
    L.lc_recover_host.argtypes = [vp, C.POINTER(vp), C.POINTER(u64), i32, u64, vp, vp, u64, vp]
    L.lc_compress_noalloc.argtypes = [vp, vp, u64, i32, vp, u64, vp]
    L.lc_debug_bins.argtypes = [vp, vp, vp, vp, vp]
    L.lc_debug_codes.argtypes = [vp, vp, vp]
    L.lc_debug_split_segments.argtypes = [C.POINTER(u64), i32, C.c_uint32, C.c_uint32, C.POINTER(C.c_uint32)]
    L.lc_debug_split_segments.restype = C.c_uint32
    L.lc_debug_decode_warps.argtypes = [i32, u64, C.c_uint32]
    L.lc_debug_decode_warps.restype = C.c_uint32
    L.lc_q4_bytes.argtypes = [u64, u64, i32]
    L.lc_q4_bytes.restype = u64
    L.lc_q4_quantize.argtypes = [vp, i32, u64, u64, u64, i32, vp, u64, vp, u64, vp]
    L.lc_recover_q4.argtypes = [vp, C.POINTER(vp), C.POINTER(u64), i32, u64, u64, i32, vp, u64, vp, vp, u64, vp]
    L.lc_q4_read.argtypes = [vp, u64, u64, u64, i32, vp, i32, u64, vp]
    L.lc_q4_matvec.argtypes = [vp, u64, u64, u64, i32, vp, i32, u64, u64, vp, i32, u64, vp]
    L.lc_debug_q4_plan.argtypes = [u64, u64, i32, i32, C.c_uint32, C.c_uint32, C.POINTER(C.c_uint32)]
    cache = C.POINTER(LCCache)
    for f in (L.lc_cache_code_bytes, L.lc_cache_scale_bytes):
        f.argtypes, f.restype = [cache], u64
    L.lc_cache_write.argtypes = L.lc_cache_read.argtypes = [vp, vp, i32, u64, vp, vp, vp]
    L.lc_cache_read_pages.argtypes = [vp, vp, i32, u64, vp, u64, C.c_uint32, C.c_uint32, vp, vp, C.c_uint32, vp, vp]
    _lib = L
    return L


def _cs(device):
    return C.c_void_p(torch.cuda.current_stream(device).cuda_stream)


def _check(rc, what):
    if rc != OK:
        raise LCError(rc, what)


def stream_bound(n: int, nbits: int) -> int:
    return int(lib().lc_stream_bound(n, nbits))


def workspace_bytes(n: int) -> int:
    return int(lib().lc_workspace_bytes(n))


def alloc_workspace(n: int, device) -> torch.Tensor:
    return torch.empty(workspace_bytes(n), dtype=torch.uint8, device=device)


def alloc_stream(n: int, nbits: int, device) -> torch.Tensor:
    return torch.empty(stream_bound(n, nbits), dtype=torch.uint8, device=device)


def _f32_cuda(t, name):
    if not (t.is_cuda and t.dtype == torch.float32 and t.is_contiguous()):
        raise ValueError("%s must be a contiguous float32 CUDA tensor" % name)
    return t


def compress_async(base, cur, nbits, stream, workspace):
    """Enqueues lc_compress on the current stream; no host synchronisation."""
    _f32_cuda(base, "base"), _f32_cuda(cur, "cur")
    if base.numel() != cur.numel():
        raise ValueError("base and cur differ in size")
    rc = lib().lc_compress(base.data_ptr(), cur.data_ptr(), base.numel(), nbits, stream.data_ptr(),
                           stream.numel(), workspace.data_ptr(), workspace.numel(), _cs(base.device))
    _check(rc, "lc_compress")


def compress_update_async(base, cur, nbits, stream, tracked_out, workspace):
    """Enqueues lc_compress_update on the current stream: the stream of lc_compress plus the advanced tracked state
    in `tracked_out` (which may be `base`); no host synchronisation."""
    _f32_cuda(base, "base"), _f32_cuda(cur, "cur"), _f32_cuda(tracked_out, "tracked_out")
    if base.numel() != cur.numel() or base.numel() != tracked_out.numel():
        raise ValueError("base, cur and tracked_out differ in size")
    rc = lib().lc_compress_update(base.data_ptr(), cur.data_ptr(), base.numel(), nbits, stream.data_ptr(),
                                  stream.numel(), tracked_out.data_ptr(), workspace.data_ptr(), workspace.numel(),
                                  _cs(base.device))
    _check(rc, "lc_compress_update")


OPT_NO_DEVICE_WAIT = 1
OPT_FIXED_WIDTH = 2
OPT_MEAN_REP = 4


def compress_opt_async(base, cur, nbits, stream, workspace, options, tracked_out=None):
    """Enqueues lc_compress_opt (``options``: 0 or OPT_NO_DEVICE_WAIT; ``tracked_out`` as for lc_compress_update)."""
    _f32_cuda(base, "base"), _f32_cuda(cur, "cur")
    rc = lib().lc_compress_opt(base.data_ptr(), cur.data_ptr(), base.numel(), nbits, stream.data_ptr(), stream.numel(),
                               None if tracked_out is None else tracked_out.data_ptr(), workspace.data_ptr(),
                               workspace.numel(), options, _cs(base.device))
    _check(rc, "lc_compress_opt")


def debug_compress_wait(base, cur, nbits, stream, workspace, spin_limit, first_ticket):
    """lc_debug_compress_wait: lc_compress with the look-back's poll limit and first tile number given."""
    rc = lib().lc_debug_compress_wait(base.data_ptr(), cur.data_ptr(), base.numel(), nbits, stream.data_ptr(),
                                      stream.numel(), workspace.data_ptr(), workspace.numel(), spin_limit,
                                      first_ticket, _cs(base.device))
    _check(rc, "lc_debug_compress_wait")


def debug_update_wait(base, cur, nbits, stream, tracked_out, workspace, spin_limit, first_ticket):
    """lc_debug_update_wait: lc_compress_update with the look-back's poll limit and first tile number given."""
    rc = lib().lc_debug_update_wait(base.data_ptr(), cur.data_ptr(), base.numel(), nbits, stream.data_ptr(),
                                    stream.numel(), tracked_out.data_ptr(), workspace.data_ptr(), workspace.numel(),
                                    spin_limit, first_ticket, _cs(base.device))
    _check(rc, "lc_debug_update_wait")


def compress_timed(base, cur, nbits, stream, workspace):
    """lc_compress with events around its kernels; returns (stats_ms, table_ms, encode_ms)."""
    ms = (C.c_float * 3)()
    rc = lib().lc_compress_timed(base.data_ptr(), cur.data_ptr(), base.numel(), nbits, stream.data_ptr(),
                                 stream.numel(), workspace.data_ptr(), workspace.numel(), _cs(base.device), ms)
    _check(rc, "lc_compress_timed")
    return tuple(float(x) for x in ms)


def last_status(workspace) -> int:
    return int(lib().lc_last_status(workspace.data_ptr(), _cs(workspace.device)))


def stream_info(stream) -> LCInfo:
    info = LCInfo()
    _check(lib().lc_stream_info(stream.data_ptr(), C.byref(info), _cs(stream.device)), "lc_stream_info")
    return info


_page = threading.local()  # page-locked host memory for lc_wait, from torch's pool and back to it with the thread


def _wait(workspace, what, stream=None):
    """Waits for the call that has just been enqueued on the current stream; raises if its status word is set. Returns
    the header of ``stream``."""
    page = getattr(_page, "tensor", None)
    if page is None:
        page = _page.tensor = torch.empty(WAIT_PAGE_BYTES, dtype=torch.uint8, device="cpu", pin_memory=True)
    info = LCInfo()
    _check(lib().lc_wait(workspace.data_ptr(), None if stream is None else stream.data_ptr(), C.byref(info), page.data_ptr(),
                         _cs(workspace.device)), what)
    return info


def compress(base, cur, nbits, stream=None, workspace=None, fixed=False, mean=False):
    """stream <- LC(cur - base). Returns the stream trimmed to its size (a view of ``stream``). ``fixed``: fixed-width
    bucket indices instead of the Huffman code (LC_OPT_FIXED_WIDTH). ``mean``: bucket means as representatives
    (LC_OPT_MEAN_REP)."""
    n = base.numel()
    if stream is None:
        stream = alloc_stream(n, nbits, base.device)
    if workspace is None:
        workspace = alloc_workspace(n, base.device)
    if fixed or mean:
        compress_opt_async(base, cur, nbits, stream, workspace, (OPT_FIXED_WIDTH if fixed else 0) | (OPT_MEAN_REP if mean else 0))
    else:
        compress_async(base, cur, nbits, stream, workspace)
    return stream[: _wait(workspace, "lc_compress (device)", stream).total_bytes]


LENGTH_CACHE_BYTES = 262144


def alloc_length_cache(device):
    """An empty length cache for compress_cached (Section 3.2, "Huffman Code Table Caching")."""
    return torch.zeros(LENGTH_CACHE_BYTES, dtype=torch.uint8, device=device)


def compress_cached_async(base, cur, nbits, stream, workspace, length_cache, tracked_out=None):
    """lc_compress_cached on the current stream; no synchronisation."""
    _f32_cuda(base, "base"), _f32_cuda(cur, "cur")
    rc = lib().lc_compress_cached(base.data_ptr(), cur.data_ptr(), base.numel(), nbits, stream.data_ptr(), stream.numel(),
                                  tracked_out.data_ptr() if tracked_out is not None else None, workspace.data_ptr(),
                                  workspace.numel(), length_cache.data_ptr(), _cs(base.device))
    _check(rc, "lc_compress_cached")


def compress_cached(base, cur, nbits, length_cache, stream=None, workspace=None, tracked_out=None):
    """stream <- LC(cur - base), code lengths taken from / stored in ``length_cache`` (changed in place)."""
    n = base.numel()
    if stream is None:
        stream = alloc_stream(n, nbits, base.device)
    if workspace is None:
        workspace = alloc_workspace(n, base.device)
    compress_cached_async(base, cur, nbits, stream, workspace, length_cache, tracked_out)
    return stream[: _wait(workspace, "lc_compress_cached (device)", stream).total_bytes]


def segments_layout(seg_begin, nbits):
    """(stream offsets, total bytes) of the streams buffer for the segments that start at ``seg_begin`` (nseg + 1
    element offsets)."""
    nseg = len(seg_begin) - 1
    sb = (C.c_uint64 * (nseg + 1))(*seg_begin)
    off = (C.c_uint64 * (nseg + 1))()
    total = int(lib().lc_segments_layout(sb, nseg, nbits, off))
    if total == 0 and nseg > 0:
        raise LCError(ERR_ARG, "lc_segments_layout")
    return [int(x) for x in off], total


def compress_segments_async(base, cur, seg_begin, nbits, streams, workspace, tracked_out=None):
    """lc_compress_segments on the current stream; no synchronisation."""
    _f32_cuda(base, "base"), _f32_cuda(cur, "cur")
    nseg = len(seg_begin) - 1
    sb = (C.c_uint64 * (nseg + 1))(*seg_begin)
    rc = lib().lc_compress_segments(base.data_ptr(), cur.data_ptr(), sb, nseg, nbits, streams.data_ptr(), streams.numel(),
                                    tracked_out.data_ptr() if tracked_out is not None else None, workspace.data_ptr(),
                                    workspace.numel(), _cs(base.device))
    _check(rc, "lc_compress_segments")


def compress_segments(base, cur, seg_begin, nbits, streams=None, workspace=None, tracked_out=None):
    """One stream per segment. Returns (streams buffer, offsets): segment i's stream starts at offsets[i]."""
    layout = None
    if streams is None:
        layout = segments_layout(seg_begin, nbits)
        streams = torch.empty(layout[1], dtype=torch.uint8, device=base.device)
    if workspace is None:
        longest = max([b - a for a, b in zip(seg_begin[:-1], seg_begin[1:])] + [0])
        workspace = alloc_workspace(longest, base.device)
    # the offsets of 62 segments take the interpreter 16 us: worked out while the GPU is busy, unless the size is needed first
    compress_segments_async(base, cur, seg_begin, nbits, streams, workspace, tracked_out)
    offsets, _ = layout or segments_layout(seg_begin, nbits)
    _wait(workspace, "lc_compress_segments (device)")
    return streams, offsets


def recover_segments_async(base, streams_list, seg_begin, nbits, out, workspace):
    """lc_recover_segments on the current stream; ``streams_list``: the buffers of a chain, in order."""
    nseg, k = len(seg_begin) - 1, len(streams_list)
    sb = (C.c_uint64 * (nseg + 1))(*seg_begin)
    ptrs = (C.c_void_p * k)(*[s.data_ptr() for s in streams_list])
    rc = lib().lc_recover_segments(base.data_ptr(), ptrs, k, sb, nseg, nbits, out.data_ptr(), workspace.data_ptr(),
                                   workspace.numel(), _cs(base.device))
    _check(rc, "lc_recover_segments")


def recover_segments(base, streams_list, seg_begin, nbits, out=None, workspace=None):
    if out is None:
        out = torch.empty_like(base)
    if workspace is None:
        workspace = alloc_workspace(0, base.device)
    recover_segments_async(base, streams_list, seg_begin, nbits, out, workspace)
    _wait(workspace, "lc_recover_segments (device)")
    return out


def compress_update(base, cur, nbits, tracked_out=None, stream=None, workspace=None):
    """stream <- LC(cur - base) and tracked_out <- base + quantized delta in one call (``tracked_out`` may be
    ``base``; allocated if None). Returns (stream trimmed to its size, tracked_out)."""
    n = base.numel()
    if stream is None:
        stream = alloc_stream(n, nbits, base.device)
    if workspace is None:
        workspace = alloc_workspace(n, base.device)
    if tracked_out is None:
        tracked_out = torch.empty_like(base)
    compress_update_async(base, cur, nbits, stream, tracked_out, workspace)
    return stream[: _wait(workspace, "lc_compress_update (device)", stream).total_bytes], tracked_out


def recover_async(base, streams, out, workspace):
    _f32_cuda(base, "base"), _f32_cuda(out, "out")
    k = len(streams)
    ptrs = (C.c_void_p * k)(*[s.data_ptr() for s in streams])
    sizes = (C.c_uint64 * k)(*[s.numel() for s in streams])
    rc = lib().lc_recover(base.data_ptr(), ptrs, sizes, k, base.numel(), out.data_ptr(), workspace.data_ptr(),
                          workspace.numel(), _cs(base.device))
    _check(rc, "lc_recover")


def recover(base, streams, out=None, workspace=None):
    """out <- base + sum of the deltas decoded from ``streams`` (applied in order)."""
    if out is None:
        out = torch.empty_like(base)
    if workspace is None:
        workspace = alloc_workspace(0, base.device)
    recover_async(base, streams, out, workspace)
    _wait(workspace, "lc_recover (device)")
    return out


def compress_two_streams(base, cur, nbits, stream, workspace, state_stream, side_stream, state_read):
    """Enqueues lc_compress_async: the statistics pass on `state_stream` (torch.cuda.Stream), then `state_read`
    (torch.cuda.Event) recorded there; table and encode on `side_stream` behind that event."""
    _f32_cuda(base, "base"), _f32_cuda(cur, "cur")
    if not state_read.cuda_event:  # torch creates the CUDA event at its first record
        state_read.record(state_stream)
    rc = lib().lc_compress_async(base.data_ptr(), cur.data_ptr(), base.numel(), nbits, stream.data_ptr(),
                                 stream.numel(), workspace.data_ptr(), workspace.numel(),
                                 C.c_void_p(state_stream.cuda_stream), C.c_void_p(side_stream.cuda_stream),
                                 C.c_void_p(state_read.cuda_event))
    _check(rc, "lc_compress_async")


STATS_BYTES = 8192


def shard_stats(base, cur, workspace, stats=None):
    """lc_shard_stats: the statistics pass of one shard; returns the 8 KB statistics buffer (uint8 tensor)."""
    _f32_cuda(base, "base"), _f32_cuda(cur, "cur")
    if stats is None:
        stats = torch.empty(STATS_BYTES, dtype=torch.uint8, device=base.device)
    _check(lib().lc_shard_stats(base.data_ptr(), cur.data_ptr(), base.numel(), stats.data_ptr(), workspace.data_ptr(),
                                workspace.numel(), _cs(base.device)), "lc_shard_stats")
    return stats


def combine_stats(buffers):
    """Element-wise combination of shards' statistics buffers on one device (what an all-reduce over the shards
    computes): counts add, the two running-maximum arrays take the unsigned maximum."""
    counts = torch.stack([b[:4096].view(torch.int64) for b in buffers]).sum(0)
    # unsigned 32-bit maximum through int64 (the words can have their top bit set)
    words = torch.stack([b[4096:].view(torch.int32).to(torch.int64) & 0xFFFFFFFF for b in buffers]).amax(0)
    out = torch.empty_like(buffers[0])
    out[:4096] = counts.view(torch.uint8)
    out[4096:] = words.to(torch.int32).view(torch.uint8)  # truncation keeps the low 32 bits
    return out


def all_reduce_stats(stats, group=None):
    """The exchange between lc_shard_stats and lc_shard_encode over a torch.distributed group: after it every rank
    holds the statistics of the whole vector. Two small all-reduces (512 sums, 1024 maxima)."""
    import torch.distributed as dist

    counts = stats[:4096].view(torch.int64).clone()
    words = stats[4096:].view(torch.int32).to(torch.int64) & 0xFFFFFFFF  # unsigned values in a signed type
    dist.all_reduce(counts, op=dist.ReduceOp.SUM, group=group)
    dist.all_reduce(words, op=dist.ReduceOp.MAX, group=group)
    stats[:4096] = counts.view(torch.uint8)
    stats[4096:] = words.to(torch.int32).view(torch.uint8)  # truncation keeps the low 32 bits
    return stats


def shard_encode(base, cur, nbits, whole_stats, workspace, stream=None):
    """lc_shard_encode: table and encode pass of one shard with the whole vector's statistics; returns the stream."""
    n = base.numel()
    if stream is None:
        stream = alloc_stream(n, nbits, base.device)
    _check(lib().lc_shard_encode(base.data_ptr(), cur.data_ptr(), n, nbits, whole_stats.data_ptr(), stream.data_ptr(),
                                 stream.numel(), workspace.data_ptr(), workspace.numel(), _cs(base.device)),
           "lc_shard_encode")
    return stream[: _wait(workspace, "lc_shard_encode (device)", stream).total_bytes]


def merge_async(base, streams, nbits, stream, scratch, workspace):
    """Enqueues lc_merge: the super-step stream of `streams` over `base` (Section 3.2, checkpoint merging)."""
    _f32_cuda(base, "base"), _f32_cuda(scratch, "scratch")
    k = len(streams)
    ptrs = (C.c_void_p * k)(*[s.data_ptr() for s in streams])
    sizes = (C.c_uint64 * k)(*[s.numel() for s in streams])
    rc = lib().lc_merge(base.data_ptr(), ptrs, sizes, k, base.numel(), nbits, stream.data_ptr(), stream.numel(),
                        scratch.data_ptr(), workspace.data_ptr(), workspace.numel(), _cs(base.device))
    _check(rc, "lc_merge")


def merge(base, streams, nbits, stream=None, scratch=None, workspace=None):
    """One stream that stands for `streams` applied to `base`: compress(base, recover(base, streams)). Returns the
    merged stream trimmed to its size; `scratch` (allocated if None) receives the recovered state."""
    n = base.numel()
    if stream is None:
        stream = alloc_stream(n, nbits, base.device)
    if scratch is None:
        scratch = torch.empty_like(base)
    if workspace is None:
        workspace = alloc_workspace(n, base.device)
    merge_async(base, streams, nbits, stream, scratch, workspace)
    return stream[: _wait(workspace, "lc_merge (device)", stream).total_bytes]


def host_arena_bytes(n, nbits, k) -> int:
    return int(lib().lc_host_arena_bytes(n, nbits, k))


def compress_host(base_cpu, cur_cpu, nbits, stream_cpu, arena):
    """Host-buffer compress: copies in, runs, copies the stream out. Returns the stream size."""
    out = C.c_uint64(0)
    rc = lib().lc_compress_host(base_cpu.data_ptr(), cur_cpu.data_ptr(), base_cpu.numel(), nbits,
                                stream_cpu.data_ptr(), stream_cpu.numel(), C.byref(out), arena.data_ptr(),
                                arena.numel(), _cs(arena.device))
    _check(rc, "lc_compress_host")
    return int(out.value)


def recover_host(base_cpu, streams_cpu, out_cpu, arena):
    k = len(streams_cpu)
    ptrs = (C.c_void_p * k)(*[s.data_ptr() for s in streams_cpu])
    sizes = (C.c_uint64 * k)(*[s.numel() for s in streams_cpu])
    rc = lib().lc_recover_host(base_cpu.data_ptr(), ptrs, sizes, k, base_cpu.numel(), out_cpu.data_ptr(),
                               arena.data_ptr(), arena.numel(), _cs(arena.device))
    _check(rc, "lc_recover_host")
    return out_cpu


def debug_bins(workspace):
    import numpy as np

    count = np.zeros(512, np.uint64)
    mmin = np.zeros(512, np.uint32)
    mmax = np.zeros(512, np.uint32)
    _check(lib().lc_debug_bins(workspace.data_ptr(), count.ctypes.data, mmin.ctypes.data, mmax.ctypes.data,
                               _cs(workspace.device)), "lc_debug_bins")
    return count, mmin, mmax


def debug_codes(workspace):
    import numpy as np

    ln = np.zeros(512, np.uint32)
    code = np.zeros(512, np.uint64)
    _check(lib().lc_debug_codes(workspace.data_ptr(), ln.ctypes.data, code.ctypes.data, _cs(workspace.device)),
           "lc_debug_codes")
    return ln, code


def compress_noalloc(base, cur, nbits, stream):
    """lc_compress_noalloc: compress with the library's built-in scratch (n <= NOALLOC_MAX_N).

    For callers that cannot allocate device memory when a snapshot is taken. Waits for the current
    stream; returns the stream trimmed to its size. Calls must not overlap on one GPU.
    """
    _f32_cuda(base, "base"), _f32_cuda(cur, "cur")
    rc = lib().lc_compress_noalloc(base.data_ptr(), cur.data_ptr(), base.numel(), nbits, stream.data_ptr(),
                                   stream.numel(), _cs(base.device))
    _check(rc, "lc_compress_noalloc")
    return stream[: stream_info(stream).total_bytes]


# ---- state in few bits: 4-bit weights and a quantised cache ------------------------------------------------------

TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
Q4_MAX_TOKENS = 1048576


# absent where torch was built without CUDA, and no tensor gets as far as a call
_raw_stream, _current_device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
_functions = {}  # of the library, by name


def _call(name, index, *args):
    """The library's ``name``(*args, the current stream of device ``index``), with that device current; raises on a host-side error.
    Small calls last as long as the interpreter takes to make them, so this does no more than that."""
    fn = _functions.get(name) or _functions.setdefault(name, getattr(lib(), name))
    if index == _current_device():
        rc = fn(*args, _raw_stream(index))
    else:
        with torch.cuda.device(index):
            rc = fn(*args, _raw_stream(index))
    if rc != OK:
        raise LCError(rc, name)


def _numbers(t, name, dims, index):
    """(LC_TYPE_*, shape, strides) of a tensor of numbers on CUDA device ``index`` whose last axis is contiguous."""
    kind, shape, strides = TYPES.get(t.dtype), t.shape, t.stride()
    if kind is None or t.get_device() != index or index < 0 or len(shape) != dims or (strides[-1] != 1 and shape[-1] > 1):
        raise ValueError("%s must be a %d-dimensional tensor of float32, bfloat16 or float16 on the CUDA device of the call, contiguous along its last axis"
                         % (name, dims))
    return kind, shape, strides


class Q4(NamedTuple):
    """A matrix of 4-bit weights: what lc_q4_quantize wrote into ``data`` (uint8), and its shape."""

    data: torch.Tensor
    rows: int
    cols: int
    group: int


def q4_bytes(rows, cols, group) -> int:
    return int(lib().lc_q4_bytes(rows, cols, group))


def alloc_q4(rows, cols, group, device) -> Q4:
    """Room for rows x cols weights, not written yet."""
    size = q4_bytes(rows, cols, group)
    if size == 0 and rows and cols:
        raise LCError(ERR_ARG, "lc_q4_bytes")
    return Q4(torch.empty(size, dtype=torch.uint8, device=device), rows, cols, group)


def q4_quantize_async(w, q4, workspace):
    """lc_q4_quantize of the matrix ``w`` into ``q4`` on the current stream; an Inf or NaN shows in last_status(workspace)."""
    data, rows, cols, group = q4
    index = data.get_device()
    kind, shape, strides = _numbers(w, "w", 2, index)
    if shape[0] != rows or shape[1] != cols:
        raise ValueError("w has another shape than the weights")
    if workspace.get_device() != index:
        raise ValueError("workspace is on another device")
    _call("lc_q4_quantize", index, w.data_ptr(), kind, rows, cols, strides[0], group, data.data_ptr(), data.numel(), workspace.data_ptr(), workspace.numel())


def q4_quantize(w, group=128, q4=None, workspace=None) -> Q4:
    """The matrix ``w`` (float32, bfloat16 or float16) as 4-bit weights; raises if it holds an Inf or NaN."""
    _numbers(w, "w", 2, w.get_device())
    if q4 is None:
        q4 = alloc_q4(w.shape[0], w.shape[1], group, w.device)
    if workspace is None:
        workspace = alloc_workspace(0, w.device)
    q4_quantize_async(w, q4, workspace)
    with torch.cuda.device(w.device):
        _wait(workspace, "lc_q4_quantize (device)")
    return q4


def recover_q4_async(base, streams, q4, scratch, workspace):
    """lc_recover_q4 on the current stream: the state that ``streams`` lead to from ``base`` (q4.rows x q4.cols values), as 4-bit
    weights. ``scratch`` receives the recovered state."""
    _f32_cuda(base, "base"), _f32_cuda(scratch, "scratch")
    if base.numel() != q4.rows * q4.cols or scratch.numel() != base.numel():
        raise ValueError("base, scratch and the weights differ in size")
    k = len(streams)
    ptrs = (C.c_void_p * k)(*[s.data_ptr() for s in streams])
    sizes = (C.c_uint64 * k)(*[s.numel() for s in streams])
    data, rows, cols, group = q4
    if not data.get_device() == base.get_device() == scratch.get_device() == workspace.get_device():
        raise ValueError("base, scratch, workspace and the weights are not on one device")
    _call("lc_recover_q4", base.get_device(), base.data_ptr(), ptrs, sizes, k, rows, cols, group, data.data_ptr(), data.numel(), scratch.data_ptr(),
          workspace.data_ptr(), workspace.numel())


def recover_q4(base, streams, rows, group=128, q4=None, scratch=None, workspace=None) -> Q4:
    """Recovers a layer of ``rows`` rows from a base and a chain of streams, as 4-bit weights."""
    if q4 is None:
        if rows < 1 or base.numel() % rows:
            raise ValueError("base does not divide into that many rows")
        q4 = alloc_q4(rows, base.numel() // rows, group, base.device)
    if scratch is None:
        scratch = torch.empty_like(base)
    if workspace is None:
        workspace = alloc_workspace(0, base.device)
    recover_q4_async(base, streams, q4, scratch, workspace)
    with torch.cuda.device(base.device):
        _wait(workspace, "lc_recover_q4 (device)")
    return q4


def q4_read(q4, out=None, dtype=torch.float32):
    """The numbers that the weights stand for, [rows, cols], on the current stream."""
    data, rows, cols, group = q4
    if out is None:
        out = torch.empty(rows, cols, dtype=dtype, device=data.device)
    index = data.get_device()
    kind, shape, strides = _numbers(out, "out", 2, index)
    if shape[0] != rows or shape[1] != cols:
        raise ValueError("out has another shape than the weights")
    _call("lc_q4_read", index, data.data_ptr(), data.numel(), rows, cols, group, out.data_ptr(), kind, strides[0])
    return out


def q4_matvec(q4, x, out=None):
    """Products of the weights with the vectors ``x`` [tokens, cols] (or one vector [cols]), on the current stream: [tokens, rows]
    in x's type, or in that of ``out`` (x's or float32). No gradient is kept."""
    if x.dim() == 1:
        return q4_matvec(q4, x.unsqueeze(0), None if out is None else out.unsqueeze(0)).squeeze(0)
    data, rows, cols, group = q4
    index = data.get_device()
    kind, shape, strides = _numbers(x, "x", 2, index)
    tokens, width = shape
    if width != cols:
        raise ValueError("x has %d columns, the weights have %d" % (width, cols))
    if x.requires_grad and torch.is_grad_enabled():
        raise ValueError("q4_matvec has no gradient: detach x, or call it under torch.no_grad()")
    if out is None:
        out, out_kind, out_stride = torch.empty(tokens, rows, dtype=x.dtype, device=x.device), kind, rows
    else:
        out_kind, out_shape, out_strides = _numbers(out, "out", 2, index)
        out_stride = out_strides[0]
        if out_shape != (tokens, rows):
            raise ValueError("out must be [tokens, rows]")
    _call("lc_q4_matvec", index, data.data_ptr(), data.numel(), rows, cols, group, x.data_ptr(), kind, tokens, strides[0], out.data_ptr(), out_kind, out_stride)
    return out


class Cache:
    """A quantised cache (lc_cache): ``codes`` [planes, slots, heads, bytes of a row] uint8 and ``scales`` [planes, slots, heads,
    groups] bfloat16, both contiguous. planes = 2: keys and values."""

    def __init__(self, codes, scales, dim, bits, group):
        if not (codes.is_cuda and codes.dtype == torch.uint8 and codes.dim() == 4 and codes.is_contiguous()):
            raise ValueError("codes must be a contiguous 4-dimensional uint8 CUDA tensor")
        if not (scales.dtype == torch.bfloat16 and scales.is_contiguous() and scales.device == codes.device):
            raise ValueError("scales must be a contiguous bfloat16 tensor beside codes")
        self.codes, self.scales, self.device = codes, scales, codes.device
        self.planes, self.slots, self.heads = codes.shape[:3]
        self.dim, self.bits, self.group = dim, bits, group
        self._c = LCCache(codes.data_ptr(), scales.data_ptr(), self.slots, self.planes, self.heads, dim, bits, group)
        self._at, self._index, self._row = C.addressof(self._c), codes.get_device(), (self.heads, dim)
        if lib().lc_cache_code_bytes(self._c) != codes.numel() or lib().lc_cache_scale_bytes(self._c) != 2 * scales.numel():
            raise ValueError("codes and scales do not have the sizes of such a cache")


def alloc_cache(slots, heads, dim, bits, group, device, planes=2) -> Cache:
    """A cache of zeros."""
    shape = LCCache(None, None, 1, 1, 1, dim, bits, group)
    row, scale = int(lib().lc_cache_code_bytes(shape)), int(lib().lc_cache_scale_bytes(shape)) // 2
    if row == 0:
        raise LCError(ERR_ARG, "lc_cache_code_bytes")
    return Cache(torch.zeros(planes, slots, heads, row, dtype=torch.uint8, device=device),
                 torch.zeros(planes, slots, heads, scale, dtype=torch.bfloat16, device=device), dim, bits, group)


_one_plane, _two_planes = struct.Struct("=QQQ").pack, struct.Struct("=QQQQQQ").pack  # an lc_rows, or two: faster than through ctypes


def _rows(cache, tensors, what):
    """The lc_rows of one tensor [rows, heads, dim] per plane, their type and their number."""
    if len(tensors) != cache.planes:
        raise ValueError("%s: the cache has %d planes" % (what, cache.planes))
    kind, shape, strides = _numbers(tensors[0], what, 3, cache._index)
    if shape[1:] != cache._row:
        raise ValueError("%s must be [rows, heads, dim] of the cache" % what)
    if cache.planes == 1:
        return _one_plane(tensors[0].data_ptr(), strides[0], strides[1]), kind, shape[0]
    kind2, shape2, strides2 = _numbers(tensors[1], what, 3, cache._index)
    if kind2 != kind or shape2 != shape:
        raise ValueError("%s: keys and values differ in shape or type" % what)
    return _two_planes(tensors[0].data_ptr(), strides[0], strides[1], tensors[1].data_ptr(), strides2[0], strides2[1]), kind, shape[0]


def _whole(t, name, dtype, index):
    if t.dtype != dtype or t.get_device() != index or not t.is_contiguous():
        raise ValueError("%s must be a contiguous %s tensor on the cache's device" % (name, dtype))
    return t.data_ptr()


def _status(status, index):
    return None if status is None else _whole(status, "status", torch.int32, index)


def alloc_status(device):
    """A status word for the cache calls, clear; last_status reads it."""
    return torch.zeros(1, dtype=torch.int32, device=device)


def cache_write(cache, k, v, slots, status=None):
    """Rows [rows, heads, dim] of keys and values (``v`` None if the cache has one plane) into the cache's ``slots`` (int64; -1: none),
    on the current stream."""
    src, kind, rows = _rows(cache, (k,) if v is None else (k, v), "keys and values")
    at = _whole(slots, "slots", torch.int64, cache._index)
    if slots.numel() != rows:
        raise ValueError("a slot for each row is needed")
    _call("lc_cache_write", cache._index, cache._at, src, kind, rows, at, _status(status, cache._index))


def _outs(cache, outs, rows, dtype):
    """The tensors that a read writes; new ones are zeroed, for rows without a slot stay as they are."""
    if outs is not None:
        return outs
    return [torch.zeros(rows, cache.heads, cache.dim, dtype=dtype, device=cache.device) for _ in range(cache.planes)]


def cache_read(cache, slots, outs=None, dtype=torch.bfloat16, status=None):
    """The rows in ``slots``, on the current stream: a tensor [rows, heads, dim] per plane (``outs``, or new ones of ``dtype``)."""
    outs = _outs(cache, outs, slots.numel(), dtype)
    out, kind, rows = _rows(cache, outs, "outs")
    at = _whole(slots, "slots", torch.int64, cache._index)
    if slots.numel() != rows:
        raise ValueError("a slot for each row is needed")
    _call("lc_cache_read", cache._index, cache._at, out, kind, rows, at, _status(status, cache._index))
    return outs


def cache_read_pages(cache, table, page, begin, outs, first=None, status=None):
    """Sequences out of pages of ``page`` slots, one behind the other, into ``outs`` (a tensor [rows, heads, dim] per plane), on the
    current stream. ``table`` [sequences, width] int32: pages; ``begin`` [sequences + 1] int32: where each sequence's rows begin in
    ``outs``; ``first`` [sequences] int32: the position of each one's first row (0 if None)."""
    index = cache._index
    out, kind, rows = _rows(cache, outs, "outs")
    if table.dim() != 2 or table.dtype != torch.int32 or table.get_device() != index or (table.shape[1] > 1 and table.stride(1) != 1):
        raise ValueError("table must be [sequences, width] int32 on the cache's device, contiguous along its last axis")
    sequences, width = table.shape
    at = _whole(begin, "begin", torch.int32, index)
    if begin.numel() != sequences + 1 or (first is not None and first.numel() != sequences):
        raise ValueError("begin has an entry per sequence and one more, first one per sequence")
    _call("lc_cache_read_pages", index, cache._at, out, kind, rows, table.data_ptr(), table.stride(0), width, page, at,
          None if first is None else _whole(first, "first", torch.int32, index), sequences, _status(status, index))
    return outs
