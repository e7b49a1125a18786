"""Python binding of libardiff (the C ABI declared in include/ardiff.h).

Argument marshalling only: every step of the hot path runs in the CUDA kernels of the shared
library. torch is used for device memory and streams. There is no CPU fallback: if the library
cannot be loaded, or a call fails, an exception is raised.

Calls are enqueued on the current stream of their tensors' device, or on `stream`. What a call reads has to
be ready on that stream, and what reads its results elsewhere has to wait for it: the caller orders the
streams. Results that a call with `stream` allocates come from that stream's memory, and tensors may be
dropped while it still runs. (Calls that write to tensors passed in alone, the head's and the gate's without
allocation, leave that to the caller.)
"""
from __future__ import annotations

import contextlib
import ctypes
import os
import struct
from typing import Dict, Optional

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libardiff.so")
_lib = None
_STAY = contextlib.nullcontext()

ARDIFF_OK = 0
ARDIFF_ERR_NULL, ARDIFF_ERR_SHAPE, ARDIFF_ERR_ALIGN, ARDIFF_ERR_UNSUPPORTED = -1, -2, -3, -4
ARDIFF_ERR_CUDA, ARDIFF_ERR_TIMEOUT, ARDIFF_ERR_NOMEM = -5, -6, -7
ARDIFF_BF16, ARDIFF_F16, ARDIFF_F32 = 0, 1, 2

_WEIGHT_FIELDS = ["Wc", "bc", "Wt1", "bt1", "Wt2", "bt2", "Win", "bin", "Wmod", "bmod",
                  "W1", "b1", "W2", "b2", "Wfm", "bfm", "Wout", "bout"]


class ArdiffError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {strerror(code)} ({code})")


class HeadDesc(ctypes.Structure):
    _fields_ = [("C", ctypes.c_int32), ("Dc", ctypes.c_int32), ("W", ctypes.c_int32),
                ("L", ctypes.c_int32), ("F", ctypes.c_int32), ("K_max", ctypes.c_int32),
                ("max_tokens", ctypes.c_int64)]


class HeadHostWeights(ctypes.Structure):
    _fields_ = [(k, ctypes.c_void_p) for k in _WEIGHT_FIELDS]


def lib() -> ctypes.CDLL:
    """Loads libardiff.so (building it with nvcc first if it is missing). Raises if it cannot."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            from . import build as _build
            _build.build()
        L = ctypes.CDLL(LIB_PATH)
        vp, i64, i32, f32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_float
        L.ardiff_strerror.restype = ctypes.c_char_p
        L.ardiff_strerror.argtypes = [ctypes.c_int]
        L.ardiff_version.restype = ctypes.c_int
        L.ardiff_last_launch_count.restype = ctypes.c_int
        L.ardiff_entropy_gate.restype = ctypes.c_int
        L.ardiff_entropy_gate.argtypes = [vp, i64, i32, f32, vp, vp, vp, vp]
        L.ardiff_entropy_gate_ex.restype = ctypes.c_int
        L.ardiff_entropy_gate_ex.argtypes = [vp, i64, i32, f32, vp, vp, vp, vp, vp]
        L.ardiff_head_create.restype = ctypes.c_int
        L.ardiff_head_create.argtypes = [ctypes.POINTER(HeadDesc), ctypes.POINTER(HeadHostWeights),
                                         ctypes.POINTER(vp)]
        L.ardiff_head_destroy.restype = ctypes.c_int
        L.ardiff_head_destroy.argtypes = [vp]
        L.ardiff_head_sample.restype = ctypes.c_int
        L.ardiff_head_sample.argtypes = [vp, vp, vp, vp, i32, vp, vp, vp, vp]
        L.ardiff_head_status.restype = ctypes.c_int
        L.ardiff_head_status.argtypes = [vp, vp]
        L.ardiff_head_set_timing.restype = ctypes.c_int
        L.ardiff_head_set_timing.argtypes = [vp, ctypes.c_int]
        L.ardiff_head_last_kernel_ms.restype = ctypes.c_int
        L.ardiff_head_last_kernel_ms.argtypes = [vp, ctypes.POINTER(ctypes.c_float)]
        L.ardiff_pipeline_create.restype = ctypes.c_int
        L.ardiff_pipeline_create.argtypes = [vp, i64, i32, i32, i32, ctypes.POINTER(vp)]
        L.ardiff_pipeline_destroy.restype = ctypes.c_int
        L.ardiff_pipeline_destroy.argtypes = [vp]
        L.ardiff_pipeline_run_host.restype = ctypes.c_int
        L.ardiff_pipeline_run_host.argtypes = [vp, vp, vp, vp, i64, f32, vp, i32, vp, vp, vp, vp]
        L.ardiff_entropy_gate_noalloc.restype = ctypes.c_int
        L.ardiff_entropy_gate_noalloc.argtypes = [vp, i64, i32, f32, vp, vp, vp, vp]
        L.ardiff_entropy_gate_stats.restype = ctypes.c_int
        L.ardiff_entropy_gate_stats.argtypes = [vp, i64, i32, f32, vp, vp, vp, vp, vp, vp]
        L.ardiff_entropy_gate_blocks.restype = ctypes.c_int
        L.ardiff_entropy_gate_blocks.argtypes = [vp, i64, i32, i32, i32, f32, vp, vp, vp, vp, vp, vp, vp]
        L.ardiff_tau_calibrate.restype = ctypes.c_int
        L.ardiff_tau_calibrate.argtypes = [vp, i64, vp, vp]
        L.ardiff_accept_prefix.restype = ctypes.c_int
        L.ardiff_accept_prefix.argtypes = [vp, vp, i64, i32, vp, vp, vp]
        L.ardiff_head_sample_coef.restype = ctypes.c_int
        L.ardiff_head_sample_coef.argtypes = [vp, vp, vp, vp, i32, vp, vp, i64, vp, vp, vp, vp]
        L.ardiff_head_last_kernel_clock.restype = ctypes.c_int
        L.ardiff_head_last_kernel_clock.argtypes = [vp, vp, ctypes.POINTER(ctypes.c_double)]
        L.ardiff_head_set_cooperative.restype = ctypes.c_int
        L.ardiff_head_set_cooperative.argtypes = [vp, ctypes.c_int]
        L.ardiff_head_few_limits.restype = ctypes.c_int
        L.ardiff_head_few_limits.argtypes = [vp, i32, ctypes.POINTER(i32), ctypes.POINTER(i32)]
        L.ardiff_head_inject_stall.restype = ctypes.c_int
        L.ardiff_head_inject_stall.argtypes = [vp, i32, ctypes.c_uint32]
        L.ardiff_head_inject_cluster_stall.restype = ctypes.c_int
        L.ardiff_head_inject_cluster_stall.argtypes = [vp, i32, ctypes.c_uint32]
        L.ardiff_pipeline_create_slots.restype = ctypes.c_int
        L.ardiff_pipeline_create_slots.argtypes = [vp, i64, i32, i32, i32, i32, ctypes.POINTER(vp)]
        L.ardiff_pipeline_submit.restype = ctypes.c_int
        L.ardiff_pipeline_submit.argtypes = [vp, i32, vp, vp, vp, i64, f32, vp, i32, vp, vp, vp, vp]
        L.ardiff_pipeline_wait.restype = ctypes.c_int
        L.ardiff_pipeline_wait.argtypes = [vp, i32]
        L.ardiff_pipeline_join.restype = ctypes.c_int
        L.ardiff_pipeline_join.argtypes = [vp, vp]
        L.ardiff_sample_tokens.restype = ctypes.c_int
        L.ardiff_sample_tokens.argtypes = [vp, i32, i64, i32, i64, vp, vp, vp, vp, vp, vp, vp, vp]
        L.ardiff_pages_extend.restype = ctypes.c_int
        L.ardiff_pages_extend.argtypes = [i32, i32, i32, vp, vp, vp, vp, i64, vp, i64, vp, vp, vp, vp, vp, vp, vp, vp]
        L.ardiff_pages_truncate.restype = ctypes.c_int
        L.ardiff_pages_truncate.argtypes = [i32, i32, i32, vp, vp, vp, vp, i64, vp, vp, vp, vp]
        L.ardiff_distill_topk.restype = ctypes.c_int
        L.ardiff_distill_topk.argtypes = [vp, i32, i64, i32, i64, vp, i32, vp, i32, f32, vp, vp, vp]
        L.ardiff_distill_topk_backward.restype = ctypes.c_int
        L.ardiff_distill_topk_backward.argtypes = [vp, i32, i64, i32, i64, vp, i32, vp, i32, f32, vp, vp, vp, i64, vp]
        L.ardiff_distill_topk_step.restype = ctypes.c_int
        L.ardiff_distill_topk_step.argtypes = [vp, i32, i64, i32, i64, vp, i32, vp, i32, f32, vp, vp, vp, vp, i64, vp]
        for fn in (L.ardiff_rotary, L.ardiff_rotary_backward, L.ardiff_rotary_append, L.ardiff_attend_pages, L.ardiff_attend_weights,
                   L.ardiff_pages_evict):
            fn.restype = ctypes.c_int
            fn.argtypes = [ctypes.c_char_p, vp]                # a packed structure, the stream
        L.ardiff_attend_workspace.restype = i64
        L.ardiff_attend_workspace.argtypes = [i32, i32, i64, i32, i32, i32]
        L.ardiff_attend_weights_workspace.restype = i64
        L.ardiff_attend_weights_workspace.argtypes = [i32]
        L.ardiff_pages_evict_workspace.restype = i64
        L.ardiff_pages_evict_workspace.argtypes = [i32, i32, i32]
        _lib = L
    return _lib


def strerror(code: int) -> str:
    return lib().ardiff_strerror(int(code)).decode()


def version() -> int:
    return int(lib().ardiff_version())


def last_launch_count() -> int:
    return int(lib().ardiff_last_launch_count())


def _check(rc: int, where: str):
    if rc != ARDIFF_OK:
        raise ArdiffError(rc, where)


def _current_stream(index: int) -> int:
    """The handle of a device's current stream."""
    import torch
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return raw(index) if raw is not None else torch.cuda.current_stream(index).cuda_stream


def _stream_ptr(stream) -> int:
    """The stream's handle; without one that of the current stream (asked for as a number where torch has that: a Stream object
    takes 2 us)."""
    import torch
    if stream is None:
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        if raw is not None:
            return raw(torch.cuda.current_device())
        stream = torch.cuda.current_stream()
    return int(stream.cuda_stream)


def _on(device):
    """with _on(device): calls go to `device`. Nothing to enter and leave where it is current already, as it mostly is."""
    import torch
    return _STAY if torch.cuda.current_device() == device.index else torch.cuda.device(device)


def _beside(fn, stream, *args):
    """fn(*args) on `stream`, for calls that allocate results. These come from that stream's memory, which nothing older on another
    stream can still be using; and every tensor is marked as used by the stream that is not its own, so that its memory is not
    given out again while a kernel reads or writes it."""
    import torch
    index = stream.device_index
    assert args[0].get_device() == index, f"a stream of cuda:{index} for tensors on {args[0].device}"
    if _current_stream(index) == stream.cuda_stream:
        return fn(*args)
    here = torch.cuda.current_stream(index)
    for t in args:
        if hasattr(t, "record_stream") and t.get_device() == index:
            t.record_stream(stream)
    with torch.cuda.stream(stream):
        out = fn(*args)
    for t in out if isinstance(out, tuple) else (out,):
        if t is not None:
            t.record_stream(here)
    return out


def ardiff_entropy_gate(feat, tau: float, mask=None, idx=None, count=None, entropy=None,
                        want_entropy: bool = False, stream=None):
    """Entropy gate + compaction on `feat` (torch bf16 CUDA tensor [n, d]).

    Returns (mask u8 [n], idx i32 [n], count i32 [1], entropy f32 [n] or None); outputs are
    allocated here unless passed in. Nothing is synchronised.
    """
    import torch
    if stream is not None:
        return _beside(ardiff_entropy_gate, stream, feat, tau, mask, idx, count, entropy, want_entropy)
    assert feat.is_cuda and feat.dtype == torch.bfloat16 and feat.dim() == 2 and feat.is_contiguous()
    n, d = feat.shape
    dev = feat.device
    if mask is None:
        mask = torch.empty((n,), dtype=torch.uint8, device=dev)
    if idx is None:
        idx = torch.empty((max(n, 1),), dtype=torch.int32, device=dev)
    if count is None:
        count = torch.empty((1,), dtype=torch.int32, device=dev)
    if entropy is None and want_entropy:
        entropy = torch.empty((n,), dtype=torch.float32, device=dev)
    with _on(dev):
        rc = lib().ardiff_entropy_gate_ex(
            feat.data_ptr(), n, d, float(tau), mask.data_ptr(), idx.data_ptr(), count.data_ptr(),
            entropy.data_ptr() if entropy is not None else None, _stream_ptr(None))
    _check(rc, "ardiff_entropy_gate")
    return mask, idx, count, entropy


def ardiff_entropy_gate_stats(feat, tau: float = -1.0, want_entropy: bool = False, stream=None):
    """Gate + threshold statistics of its own entropies in one pass. Returns (mask, idx, count, entropy or
    None, out3 float64 CUDA tensor [3] = mean, std, 0.3 mean - 0.1 std)."""
    import torch
    if stream is not None:
        return _beside(ardiff_entropy_gate_stats, stream, feat, tau, want_entropy)
    assert feat.is_cuda and feat.dtype == torch.bfloat16 and feat.dim() == 2 and feat.is_contiguous()
    n, d = feat.shape
    dev = feat.device
    mask = torch.empty((n,), dtype=torch.uint8, device=dev)
    idx = torch.empty((max(n, 1),), dtype=torch.int32, device=dev)
    count = torch.empty((1,), dtype=torch.int32, device=dev)
    entropy = torch.empty((n,), dtype=torch.float32, device=dev) if want_entropy else None
    out3 = torch.empty((3,), dtype=torch.float64, device=dev)
    fn = lib().ardiff_entropy_gate_stats
    with _on(dev):
        rc = fn(feat.data_ptr(), n, d, float(tau), mask.data_ptr(), idx.data_ptr(), count.data_ptr(),
                entropy.data_ptr() if entropy is not None else None, out3.data_ptr(), _stream_ptr(None))
    _check(rc, "ardiff_entropy_gate_stats")
    return mask, idx, count, entropy, out3


def ardiff_entropy_gate_blocks(feat, rows_per_token: int, gamma: int, tau: float, want_token_entropy: bool = False,
                               want_row_entropy: bool = True, stream=None):
    """Block-prefix gate (early stop inside draft blocks of `gamma` tokens, each token owning
    `rows_per_token` rows of feat). Returns (mask u8 [n], idx i32 [n], count i32 [1], block_len i32
    [ceil(n/gamma)], row_entropy f32 [n*rows_per_token], token_entropy f32 [n] or None)."""
    import torch
    if stream is not None:
        return _beside(ardiff_entropy_gate_blocks, stream, feat, rows_per_token, gamma, tau, want_token_entropy, want_row_entropy)
    assert feat.is_cuda and feat.dtype == torch.bfloat16 and feat.dim() == 2 and feat.is_contiguous()
    rows, d = feat.shape
    assert rows % rows_per_token == 0
    n = rows // rows_per_token
    dev = feat.device
    fn = lib().ardiff_entropy_gate_blocks
    mask = torch.empty((n,), dtype=torch.uint8, device=dev)
    idx = torch.empty((max(n, 1),), dtype=torch.int32, device=dev)
    count = torch.empty((1,), dtype=torch.int32, device=dev)
    block_len = torch.empty((max((n + gamma - 1) // gamma, 1),), dtype=torch.int32, device=dev)
    row_ent = torch.empty((max(rows, 1),), dtype=torch.float32, device=dev) if want_row_entropy else None
    tok_ent = torch.empty((max(n, 1),), dtype=torch.float32, device=dev) if want_token_entropy else None
    with _on(dev):
        rc = fn(feat.data_ptr(), n, rows_per_token, d, gamma, float(tau),
                row_ent.data_ptr() if row_ent is not None else None,
                tok_ent.data_ptr() if tok_ent is not None else None, mask.data_ptr(), idx.data_ptr(),
                count.data_ptr(), block_len.data_ptr(), _stream_ptr(None))
    _check(rc, "ardiff_entropy_gate_blocks")
    return mask, idx, count, block_len, row_ent, tok_ent


def ardiff_tau_calibrate(entropy, stream=None):
    """(mean, std, tau = 0.3 mean - 0.1 std) of a float32 CUDA tensor of entropies, as a float64 CUDA tensor [3]."""
    import torch
    if stream is not None:
        return _beside(ardiff_tau_calibrate, stream, entropy)
    assert entropy.is_cuda and entropy.dtype == torch.float32 and entropy.is_contiguous()
    out = torch.empty((3,), dtype=torch.float64, device=entropy.device)
    fn = lib().ardiff_tau_calibrate
    with _on(entropy.device):
        rc = fn(entropy.data_ptr(), entropy.numel(), out.data_ptr(), _stream_ptr(None))
    _check(rc, "ardiff_tau_calibrate")
    return out


def ardiff_accept_prefix(r, ratio, gamma: int, block_len=None, stream=None):
    """Accepted draft length per block of `gamma`: first position with r > ratio, else the length of the
    draft (block_len[b] tokens where the early stop truncated block b; the whole block if block_len is None)."""
    import torch
    if stream is not None:
        return _beside(ardiff_accept_prefix, stream, r, ratio, gamma, block_len)
    assert r.is_cuda and r.dtype == torch.float32 and ratio.dtype == torch.float32 and r.shape == ratio.shape
    n = r.numel()
    nb = (n + gamma - 1) // gamma
    out = torch.empty((max(nb, 1),), dtype=torch.int32, device=r.device)
    if block_len is not None:
        assert block_len.is_cuda and block_len.dtype == torch.int32 and block_len.numel() >= nb
    fn = lib().ardiff_accept_prefix
    with _on(r.device):
        rc = fn(r.data_ptr(), ratio.data_ptr(), n, gamma, block_len.data_ptr() if block_len is not None else None,
                out.data_ptr(), _stream_ptr(None))
    _check(rc, "ardiff_accept_prefix")
    return out[:(n + gamma - 1) // gamma]


class _Torch:
    """What the calls below ask of torch every time, looked up once (they take microseconds in all, so lookups count)."""

    def __init__(self):
        import torch
        self.i32, self.i64, self.f32 = torch.int32, torch.int64, torch.float32
        self.types = {torch.bfloat16: ARDIFF_BF16, torch.float16: ARDIFF_F16, torch.float32: ARDIFF_F32}
        self.u8 = torch.uint8
        self.empty, self.empty_like, self.device = torch.empty, torch.empty_like, torch.cuda.device
        self.current = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
        self.stream = getattr(torch._C, "_cuda_getCurrentRawStream", lambda i: torch.cuda.current_stream(i).cuda_stream)


_torch = None


def _t() -> _Torch:
    global _torch
    if _torch is None:
        _torch = _Torch()
    return _torch


def _run(fn, where: str, index: int, *args):
    """fn(*args, current stream) with the device of the tensors current; raises on an error."""
    t = _torch
    if t.current() == index:
        rc = fn(*args, t.stream(index))
    else:
        with t.device(index):
            rc = fn(*args, t.stream(index))
    if rc:
        raise ArdiffError(rc, where)


def _ptr(t):
    return None if t is None else t.data_ptr()


# The C calls take these sizes as int32, and ctypes would cut off what does not fit.
_SIZES = 2**31
_TOO_LARGE = "sizes that do not fit 32 bits"


def _rows(x) -> int:
    """Distance of the rows of a matrix whose rows are contiguous (one row, or one column, may have any)."""
    n, V = x.shape
    assert V < _SIZES, _TOO_LARGE
    if x.is_contiguous():
        return V
    assert V <= 1 or x.stride(1) == 1, "rows must be contiguous"
    ld = x.stride(0) if n > 1 else V
    assert ld >= V, "rows must not overlap"
    return ld


def _check_i32(x, n: int, index: int):
    assert x.dtype is _torch.i32 and x.numel() == n and x.get_device() == index and x.is_contiguous(), \
        f"int32 tensor of {n} entries on cuda:{index} expected, got {x.dtype} {tuple(x.shape)} on {x.device}"


def _check_f32(x, n: int, index: int):
    assert x.dtype is _torch.f32 and x.numel() == n and x.get_device() == index and x.is_contiguous(), \
        f"float32 tensor of {n} entries on cuda:{index} expected, got {x.dtype} {tuple(x.shape)} on {x.device}"


def ardiff_sample_tokens(logits, u, temperature=None, top_k=None, top_p=None, min_p=None, token=None, logprob=None, stream=None):
    """The next token of every row of logits [n, V] (bf16, f16 or f32 CUDA tensor, rows contiguous) by the uniform numbers u
    (f32 [n], 0 <= u < 1). temperature, top_p, min_p (f32 [n]) and top_k (int32 [n]) are every row's own, or None (off).
    Returns (token int32 [n], logprob f32 [n]); -1 and NaN for rows that have no softmax or bad settings."""
    if stream is not None:
        return _beside(ardiff_sample_tokens, stream, logits, u, temperature, top_k, top_p, min_p, token, logprob)
    t = _t()
    n, V = logits.shape
    index = logits.get_device()
    assert index >= 0
    for x in (u, temperature, top_p, min_p):
        if x is not None:
            _check_f32(x, n, index)
    if top_k is not None:
        _check_i32(top_k, n, index)
    if token is None:
        token = t.empty((n,), dtype=t.i32, device=logits.device)
    else:
        _check_i32(token, n, index)
    if logprob is None:
        logprob = t.empty((n,), dtype=t.f32, device=logits.device)
    else:
        _check_f32(logprob, n, index)
    _run(lib().ardiff_sample_tokens, "ardiff_sample_tokens", index, logits.data_ptr(), t.types.get(logits.dtype, -1), n, V,
         _rows(logits), u.data_ptr(), _ptr(temperature), _ptr(top_k), _ptr(top_p), _ptr(min_p), token.data_ptr(), logprob.data_ptr())
    return token, logprob


def _pages_args(length, other, table, free_pages, free_count, page):
    R, width = table.shape
    assert R < _SIZES and width < _SIZES and -_SIZES <= page < _SIZES, _TOO_LARGE
    index = length.get_device()
    assert index >= 0
    _check_i32(length, R, index)
    _check_i32(other, R, index)
    _check_i32(table, R * width, index)
    _check_i32(free_pages, free_pages.numel(), index)
    _check_i32(free_count, 1, index)
    return R, width, index


def _made_i32(x, n: int, like):
    if x is None:
        return _torch.empty((n,), dtype=_torch.i32, device=like.device)
    _check_i32(x, n, like.get_device())
    return x


def ardiff_pages_extend(length, add, table, free_pages, free_count, page: int, slot, position=None, request=None, offset=None,
                        new_length=None, new_free_count=None, status=None, stream=None):
    """add[r] new tokens for request r of a paged cache: pages from the end of the free list, the block table lengthened in
    place, slot / position / request of every new token (as many as fit in slot; position and request are written if
    passed). int32 CUDA tensors, slot int64. new_length may be `length` and new_free_count `free_count`; what is not passed is
    allocated. Returns (offset [R + 1], new_length [R], new_free_count [1], status [1]); status is not looked at here."""
    if stream is not None:
        return _beside(ardiff_pages_extend, stream, length, add, table, free_pages, free_count, page, slot, position, request, offset,
                       new_length, new_free_count, status)
    t = _t()
    R, width, index = _pages_args(length, add, table, free_pages, free_count, page)
    tokens = slot.numel()
    assert slot.dtype is t.i64 and slot.get_device() == index and slot.is_contiguous()
    if position is not None:
        _check_i32(position, tokens, index)
    if request is not None:
        _check_i32(request, tokens, index)
    offset = _made_i32(offset, R + 1, length)
    new_length = _made_i32(new_length, R, length)
    new_free_count = _made_i32(new_free_count, 1, length)
    status = _made_i32(status, 1, length)
    _run(lib().ardiff_pages_extend, "ardiff_pages_extend", index, R, page, width, length.data_ptr(), add.data_ptr(),
         table.data_ptr(), free_pages.data_ptr(), free_pages.numel(), free_count.data_ptr(), tokens, slot.data_ptr(), _ptr(position),
         _ptr(request), offset.data_ptr(), new_length.data_ptr(), new_free_count.data_ptr(), status.data_ptr())
    return offset, new_length, new_free_count, status


def ardiff_pages_truncate(length, target, table, free_pages, free_count, page: int, new_free_count=None, status=None,
                          stream=None):
    """Leaves request r of a paged cache its first target[r] tokens; the pages that none of them needs go back to the free list
    (in place). int32 CUDA tensors; new_free_count may be `free_count`. Returns (new_free_count [1], status [1])."""
    if stream is not None:
        return _beside(ardiff_pages_truncate, stream, length, target, table, free_pages, free_count, page, new_free_count, status)
    _t()
    R, width, index = _pages_args(length, target, table, free_pages, free_count, page)
    new_free_count = _made_i32(new_free_count, 1, length)
    status = _made_i32(status, 1, length)
    _run(lib().ardiff_pages_truncate, "ardiff_pages_truncate", index, R, page, width, length.data_ptr(), target.data_ptr(),
         table.data_ptr(), free_pages.data_ptr(), free_pages.numel(), free_count.data_ptr(), new_free_count.data_ptr(),
         status.data_ptr())
    return new_free_count, status


def _distill_args(logits, teacher, ids):
    t = _t()
    n, V = logits.shape
    k = teacher.shape[1]
    assert k < _SIZES, _TOO_LARGE
    index = logits.get_device()
    assert index >= 0 and teacher.get_device() == index and teacher.is_contiguous() and teacher.shape[0] == n
    assert ids.shape == teacher.shape, f"ids of {tuple(teacher.shape)} expected, got {tuple(ids.shape)}"
    _check_i32(ids, n * k, index)
    return index, (logits.data_ptr(), t.types.get(logits.dtype, -1), n, V, _rows(logits), teacher.data_ptr(),
                   t.types.get(teacher.dtype, -1), ids.data_ptr(), k)


def _made_f32(x, shape, n: int, like):
    if x is None:
        return _torch.empty(shape, dtype=_torch.f32, device=like.device)
    _check_f32(x, n, like.get_device())
    return x


def _made_grad(grad, logits):
    if grad is None:
        return _torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
    assert grad.dtype is logits.dtype and grad.get_device() == logits.get_device() and grad.shape == logits.shape
    return grad


def ardiff_distill_topk(logits, teacher, ids, temperature: float = 1.0, loss=None, stats=None, stream=None):
    """Divergence of every row of a student's logits [n, V] (bf16, f16 or f32, rows contiguous) from the softmax of the teacher's
    entries (teacher [n, k] at ids [n, k] int32; ids outside 0 .. V - 1 are no entries).
    Returns (loss f32 [n], stats f32 [n, 2]: what ardiff_distill_topk_backward needs of the rows)."""
    if stream is not None:
        return _beside(ardiff_distill_topk, stream, logits, teacher, ids, temperature, loss, stats)
    index, args = _distill_args(logits, teacher, ids)
    n = logits.shape[0]
    loss, stats = _made_f32(loss, (n,), n, logits), _made_f32(stats, (n, 2), 2 * n, logits)
    _run(lib().ardiff_distill_topk, "ardiff_distill_topk", index, *args, temperature, loss.data_ptr(), stats.data_ptr())
    return loss, stats


def ardiff_distill_topk_backward(logits, teacher, ids, stats, weight, temperature: float = 1.0, grad=None, stream=None):
    """Gradient of sum(weight * loss) with respect to the logits, from the stats that ardiff_distill_topk gave for the same
    inputs; in the logits' type. `grad` may be `logits`."""
    if stream is not None:
        return _beside(ardiff_distill_topk_backward, stream, logits, teacher, ids, stats, weight, temperature, grad)
    index, args = _distill_args(logits, teacher, ids)
    n = logits.shape[0]
    _check_f32(stats, 2 * n, index)
    _check_f32(weight, n, index)
    grad = _made_grad(grad, logits)
    _run(lib().ardiff_distill_topk_backward, "ardiff_distill_topk_backward", index, *args, temperature, stats.data_ptr(),
         weight.data_ptr(), grad.data_ptr(), _rows(grad))
    return grad


def ardiff_distill_topk_step(logits, teacher, ids, weight, temperature: float = 1.0, loss=None, stats=None, grad=None,
                             stream=None):
    """Loss, stats and the gradient of sum(weight * loss) in one pass. `grad` may be `logits`. Returns (loss, stats, grad)."""
    if stream is not None:
        return _beside(ardiff_distill_topk_step, stream, logits, teacher, ids, weight, temperature, loss, stats, grad)
    index, args = _distill_args(logits, teacher, ids)
    n = logits.shape[0]
    _check_f32(weight, n, index)
    grad = _made_grad(grad, logits)
    loss, stats = _made_f32(loss, (n,), n, logits), _made_f32(stats, (n, 2), 2 * n, logits)
    _run(lib().ardiff_distill_topk_step, "ardiff_distill_topk_step", index, *args, temperature, weight.data_ptr(),
         loss.data_ptr(), stats.data_ptr(), grad.data_ptr(), _rows(grad))
    return loss, stats, grad


# The structures that these calls take, all of 64-bit fields: packed at once, where ctypes takes a tenth of a microsecond an argument.
_ROTARY, _APPEND = struct.Struct("24q"), struct.Struct("36q")
_ATTEND, _WEIGHTS, _EVICT = struct.Struct("27qd9q"), struct.Struct("24q2d6q"), struct.Struct("32q")


def _at(t) -> int:
    return 0 if t is None else t.data_ptr()


def _made_like(x):
    """A contiguous result of x's shape and type (empty_like takes half the time of empty, but keeps the order of strides)."""
    return _torch.empty_like(x) if x.is_contiguous() else _torch.empty(x.shape, dtype=x.dtype, device=x.device)


def _heads(x, index: int):
    """Address, strides of tokens and heads, and heads of a tensor [n, heads, width] whose rows are contiguous."""
    n, heads, width = x.shape
    token, head, one = x.stride()
    assert x.get_device() == index and (one == 1 or width <= 1), f"a tensor on cuda:{index} with contiguous rows expected"
    return x.data_ptr(), token, head, heads


def _out_heads(x, like, index: int):
    """The same without the number of heads, for results of the shape and type of `like`. They must not overlap themselves."""
    assert x.dtype is like.dtype and x.shape == like.shape, f"{like.dtype} {tuple(like.shape)} expected, got {x.dtype} {tuple(x.shape)}"
    n, heads, width = x.shape
    token, head, one = x.stride()
    assert x.get_device() == index and (one == 1 or width <= 1), f"a tensor on cuda:{index} with contiguous rows expected"
    assert (heads <= 1 or head >= width) and (n <= 1 or token >= width) and \
        (heads <= 1 or n <= 1 or (token >= (heads - 1) * head + width if token >= head else head >= (n - 1) * token + width)), "rows of results must not overlap"
    return x.data_ptr(), token, head


def _rotary_args(q, k, position, freq, axis):
    t = _t()
    index = q.get_device()
    n, _, width = q.shape
    assert index >= 0 and k.dtype is q.dtype and k.shape[0] == n and k.shape[2] == width, "queries and keys of the same tokens, type and width expected"
    if position.dim() == 1:
        position = position[None]
    axes = position.shape[0]
    assert position.dtype is t.i32 and position.get_device() == index and position.shape[1] == n and (n <= 1 or position.stride(1) == 1), \
        f"int32 positions [axes, {n}] on cuda:{index} expected"
    pairs = freq.numel()
    _check_f32(freq, pairs, index)
    if axis is not None:
        _check_i32(axis, pairs, index)
    return index, t.types.get(q.dtype, -1), n, width, (position.data_ptr(), position.stride(0) if axes > 1 else 0, axes, freq.data_ptr(), _at(axis), pairs)


def _turned(fn, where, q, k, position, freq, axis, neighbours, q_out, k_out):
    index, dtype, n, width, angles = _rotary_args(q, k, position, freq, axis)
    if q_out is None:
        q_out = _made_like(q)
    if k_out is None:
        k_out = _made_like(k)
    qp, qt, qh, q_heads = _heads(q, index)
    kp, kt, kh, k_heads = _heads(k, index)
    _run(fn, where, index, _ROTARY.pack(qp, qt, qh, *_out_heads(q_out, q, index), q_heads, kp, kt, kh, *_out_heads(k_out, k, index), k_heads,
                                        dtype, n, width, *angles, 1 if neighbours else 0))
    return q_out, k_out


def ardiff_rotary(q, k, position, freq, axis=None, neighbours: bool = False, q_out=None, k_out=None, stream=None):
    """Queries [n, heads, width] and keys [n, kv heads, width] (bf16, f16 or f32, any strides with contiguous rows) turned by their positions:
    pair i of token t by position[axis[i], t] * freq[i] (position int32 [axes, n] or [n], freq f32 [pairs], axis int32 [pairs] or None for the
    first). A pair is values i and i + pairs, or 2 i and 2 i + 1 (neighbours); values from 2 * pairs on are copied. q_out and k_out may be q and k.
    Returns (q_out, k_out)."""
    if stream is not None:
        return _beside(ardiff_rotary, stream, q, k, position, freq, axis, neighbours, q_out, k_out)
    return _turned(lib().ardiff_rotary, "ardiff_rotary", q, k, position, freq, axis, neighbours, q_out, k_out)


def ardiff_rotary_backward(grad_q, grad_k, position, freq, axis=None, neighbours: bool = False, q_out=None, k_out=None, stream=None):
    """Gradients with respect to what ardiff_rotary was given, from those with respect to what it returned. Arguments as there."""
    if stream is not None:
        return _beside(ardiff_rotary_backward, stream, grad_q, grad_k, position, freq, axis, neighbours, q_out, k_out)
    return _turned(lib().ardiff_rotary_backward, "ardiff_rotary_backward", grad_q, grad_k, position, freq, axis, neighbours, q_out, k_out)


def _cache_args(cache, dtype, index: int):
    """Address and strides of pages, tokens and heads of a cache [pages, page, heads, width] whose rows are contiguous."""
    a, b, c, d = cache.stride()
    assert cache.dtype is dtype and cache.get_device() == index and (d == 1 or cache.shape[3] <= 1), \
        f"a cache of {dtype} on cuda:{index} with contiguous rows expected"
    return cache.data_ptr(), a, b, c


def _written_cache_args(cache, dtype, index: int):
    """The same for a cache that is written: no two of its rows may be one (torch refuses to write to those, too)."""
    args = _cache_args(cache, dtype, index)
    if 0 in args[1:]:
        assert all(s or n <= 1 for s, n in zip(args[1:], cache.shape)), "rows of a cache that is written must not be one another's"
    return args


def ardiff_rotary_append(q, k, v, position, freq, slot, k_cache, v_cache, axis=None, count=None, neighbours: bool = False, q_out=None,
                         stream=None):
    """Queries turned as by ardiff_rotary (into q_out), keys turned and written with their values into a cache (k_cache, v_cache [pages, page,
    kv heads, width], rows contiguous) at slot[t] (int64 [n]: page * id + place, as ardiff_pages_extend lists them; others are not written).
    Tokens from count[0] on (int32 [1], e.g. offset[-1:]) are not touched. Returns q_out."""
    if stream is not None:
        return _beside(ardiff_rotary_append, stream, q, k, v, position, freq, slot, k_cache, v_cache, axis, count, neighbours, q_out)
    index, dtype, n, width, angles = _rotary_args(q, k, position, freq, axis)
    if q_out is None:
        q_out = _made_like(q)
    assert v.shape == k.shape and v.dtype is k.dtype, "keys and values of the same shape and type expected"
    assert slot.dtype is _torch.i64 and slot.numel() == n and slot.get_device() == index and slot.is_contiguous(), f"int64 slots [{n}] on cuda:{index} expected"
    if count is not None:
        _check_i32(count, 1, index)
    pages, page = k_cache.shape[:2]
    assert k_cache.shape == v_cache.shape and k_cache.shape[2] == k.shape[1] and k_cache.shape[3] == width, "caches [pages, page, kv heads, width] expected"
    qp, qt, qh, q_heads = _heads(q, index)
    kp, kt, kh, k_heads = _heads(k, index)
    _run(lib().ardiff_rotary_append, "ardiff_rotary_append", index,
         _APPEND.pack(qp, qt, qh, *_out_heads(q_out, q, index), q_heads, kp, kt, kh, *_heads(v, index)[:3], k_heads, dtype, n, width, *angles,
                      1 if neighbours else 0, slot.data_ptr(), _at(count), *_written_cache_args(k_cache, k.dtype, index),
                      *_written_cache_args(v_cache, k.dtype, index), pages, page))
    return q_out


def _attend_args(q, k_cache, table, length, offset):
    t = _t()
    R, width = table.shape
    pages, page, heads, D = k_cache.shape
    T, q_heads, _ = q.shape
    assert R < _SIZES and T < _SIZES and q_heads < _SIZES and heads < _SIZES and D < _SIZES, _TOO_LARGE
    index = q.get_device()
    assert index >= 0 and q.shape[2] == D, "queries and keys of the same width expected"
    _check_i32(table, R * width, index)
    _check_i32(length, R, index)
    _check_i32(offset, R + 1, index)
    return index, R, width, pages, page, heads, D, T, t.types.get(q.dtype, -1)


def _workspace(size: int, where: str, device):
    if size < 0:
        raise ArdiffError(size, where)
    return _torch.empty((size,), dtype=_torch.u8, device=device)


def ardiff_attend_pages(q, k_cache, v_cache, table, length, offset, group=None, shared=None, most=None, scale=None, causal: bool = True,
                        out=None, lse=None, status=None, stream=None):
    """Attention of every request's new tokens (rows offset[r] .. offset[r + 1] - 1 of q [tokens, heads, width], bf16 or f16) over its length[r]
    tokens, the new ones at their end, in the pages table[r] of the caches [pages, page, kv heads, width]. Requests group[g] .. group[g + 1] - 1
    share their first shared[g] tokens, which are read once for all of them (int32 [groups + 1] and [groups]). most: new tokens of a request at
    most, if known. scale: 1 / sqrt(width) unless given. Returns (out like q, lse f32 [tokens, heads], status int32 [1], not looked at here); rows behind
    offset[-1] are left as they were."""
    if stream is not None:
        return _beside(ardiff_attend_pages, stream, q, k_cache, v_cache, table, length, offset, group, shared, most, scale, causal, out, lse, status)
    index, R, width, pages, page, heads, D, T, dtype = _attend_args(q, k_cache, table, length, offset)
    assert k_cache.shape == v_cache.shape, "caches of the same shape expected"
    assert (group is None) == (shared is None), "group and shared belong together"
    groups = 0
    if group is not None:
        groups = shared.numel()
        assert groups < _SIZES, _TOO_LARGE
        _check_i32(group, groups + 1, index)
        _check_i32(shared, groups, index)
    if out is None:
        out = _made_like(q)
    qp, qt, qh, q_heads = _heads(q, index)
    lse = _made_f32(lse, (T, q_heads), T * q_heads, q)
    status = _made_i32(status, 1, length)
    L = lib()
    size = L.ardiff_attend_workspace(R, groups, T, q_heads, heads, D)
    work = _workspace(size, "ardiff_attend_pages", q.device)
    _run(L.ardiff_attend_pages, "ardiff_attend_pages", index,
         _ATTEND.pack(qp, qt, qh, q_heads, T, dtype, *_cache_args(k_cache, q.dtype, index), *_cache_args(v_cache, q.dtype, index), pages, page,
                      heads, D, table.data_ptr(), width, R, length.data_ptr(), offset.data_ptr(), groups, _at(group), _at(shared),
                      0 if most is None else most, D ** -0.5 if scale is None else scale, 1 if causal else 0, *_out_heads(out, q, index),
                      lse.data_ptr(), q_heads, status.data_ptr(), work.data_ptr(), size))
    return out, lse, status


def _scores(x, R: int, index: int) -> int:
    """Distance of the rows of a matrix of R rows; its row length may be any."""
    assert x.dim() == 2 and x.shape[0] == R and x.get_device() == index, f"{R} rows on cuda:{index} expected"
    if x.is_contiguous():
        return x.shape[1]
    assert x.shape[1] <= 1 or x.stride(1) == 1, "rows must be contiguous"
    assert x.stride(0) >= x.shape[1], "rows must not overlap"
    return x.stride(0)


def ardiff_attend_weights(q, k_cache, table, length, offset, lse, score, first=None, decay: float = 1.0, scale=None,
                          causal: bool = True, new_score=None, status=None, stream=None):
    """The attention weight that every token got from the new tokens' queries, added to decay * score (f32 [requests, places]): arguments as for
    ardiff_attend_pages, whose lse it takes. Places below first[r] (int32 [requests]) and from length[r] on are left as they are in new_score, which may
    be `score` (and is made without them being set if not given). Returns (new_score, status int32 [1])."""
    if stream is not None:
        return _beside(ardiff_attend_weights, stream, q, k_cache, table, length, offset, lse, score, first, decay, scale, causal, new_score, status)
    index, R, width, pages, page, heads, D, T, dtype = _attend_args(q, k_cache, table, length, offset)
    qp, qt, qh, q_heads = _heads(q, index)
    _check_f32(lse, T * q_heads, index)
    if first is not None:
        _check_i32(first, R, index)
    ld = _scores(score, R, index)
    if new_score is None:
        new_score = _torch.empty(score.shape, dtype=_torch.f32, device=score.device)
    assert score.dtype is _torch.f32 and new_score.dtype is _torch.f32 and new_score.shape == score.shape, "f32 scores of the same shape expected"
    new_ld = _scores(new_score, R, index)
    places = score.shape[1]
    assert width * page <= places, f"scores for the {width * page} places of a row of the table expected, got {places}"
    status = _made_i32(status, 1, length)
    L = lib()
    size = L.ardiff_attend_weights_workspace(R)
    work = _workspace(size, "ardiff_attend_weights", q.device)
    _run(L.ardiff_attend_weights, "ardiff_attend_weights", index,
         _WEIGHTS.pack(qp, qt, qh, q_heads, T, dtype, *_cache_args(k_cache, q.dtype, index), pages, page, heads, D, table.data_ptr(), width, R,
                       length.data_ptr(), offset.data_ptr(), _at(first), lse.data_ptr(), q_heads, score.data_ptr(), ld,
                       D ** -0.5 if scale is None else scale, decay, 1 if causal else 0, new_score.data_ptr(), new_ld, status.data_ptr(),
                       work.data_ptr(), size))
    return new_score, status


def ardiff_pages_evict(length, budget, score, table, k_cache, v_cache, first=None, position=None, seen=None, recent: int = 0, new_length=None,
                       new_score=None, new_position=None, source=None, status=None, stream=None):
    """Leaves request r its budget[r] tokens of largest score (f32 [requests, places]), those below first[r] and those whose position (int32 [requests,
    places], or the place) is at or above seen[r] - recent before all others. Kept tokens behind the new end move, in the caches too, into the places
    that became free. int32 CUDA tensors [requests]; new_length may be `length`, new_score `score`, new_position `position`; source (int32, like
    score): the place that every token had. Entries behind the new length are left as they are (not set where made here). Returns
    (new_length, new_score, new_position or None, status)."""
    if stream is not None:
        return _beside(ardiff_pages_evict, stream, length, budget, score, table, k_cache, v_cache, first, position, seen, recent, new_length,
                       new_score, new_position, source, status)
    t = _t()
    R, width = table.shape
    pages, page, heads, D = k_cache.shape
    assert R < _SIZES and width < _SIZES and page < _SIZES, _TOO_LARGE
    index = length.get_device()
    assert index >= 0 and k_cache.shape == v_cache.shape, "caches of the same shape expected"
    _check_i32(table, R * width, index)
    for x in (length, budget, first, seen):
        if x is not None:
            _check_i32(x, R, index)
    new_length = _made_i32(new_length, R, length)
    ld = _scores(score, R, index)
    places = score.shape[1]
    if new_score is None:
        new_score = t.empty(score.shape, dtype=t.f32, device=score.device)
    if new_position is None and position is not None:
        new_position = t.empty(score.shape, dtype=t.i32, device=score.device)
    assert score.dtype is t.f32 and new_score.dtype is t.f32 and new_score.shape == score.shape, "f32 scores of the same shape expected"
    assert width * page <= places, f"scores for the {width * page} places of a row of the table expected, got {places}"
    new_ld = _scores(new_score, R, index)
    for x, rows in ((position, ld), (new_position, new_ld), (source, new_ld)):
        if x is not None:
            assert x.dtype is t.i32 and x.shape == score.shape and _scores(x, R, index) == rows, "int32 positions laid out as the scores are expected"
    status = _made_i32(status, 1, length)
    L = lib()
    size = L.ardiff_pages_evict_workspace(R, page, width)
    work = _workspace(size, "ardiff_pages_evict", length.device)
    _run(L.ardiff_pages_evict, "ardiff_pages_evict", index,
         _EVICT.pack(R, length.data_ptr(), budget.data_ptr(), _at(first), score.data_ptr(), ld, _at(position), _at(seen), recent,
                     table.data_ptr(), width, t.types.get(k_cache.dtype, -1), *_written_cache_args(k_cache, k_cache.dtype, index),
                     *_written_cache_args(v_cache, k_cache.dtype, index), pages, page, heads, D, new_length.data_ptr(), new_score.data_ptr(),
                     _at(new_position), _at(source), new_ld, status.data_ptr(), work.data_ptr(), size))
    return new_length, new_score, new_position, status


GATE_NOALLOC_MAX_BLOCKS = 1024
GATE_NOALLOC_MAX_TOKENS = 1 << 24


def ardiff_entropy_gate_noalloc(feat, tau: float, mask, idx, count, stream=None):
    """The gate for callers that may not allocate device memory (a process whose own pool owns the
    device, code inside a stream capture, a latency-critical loop): same kernels and results as
    ardiff_entropy_gate, but the library's scratch is a fixed __device__ array instead of a
    cudaMalloc on first use. Because nothing may be allocated, the caller passes every output
    (mask u8 [n], idx i32 [n], count i32 [1]); there is no entropy output. n is limited to
    GATE_NOALLOC_MAX_TOKENS. Calls on one device share the scratch: do not let two overlap."""
    import torch
    assert feat.is_cuda and feat.dtype == torch.bfloat16 and feat.dim() == 2 and feat.is_contiguous()
    fn = lib().ardiff_entropy_gate_noalloc
    n, d = feat.shape
    with _on(feat.device):
        rc = fn(feat.data_ptr(), n, d, float(tau), mask.data_ptr(), idx.data_ptr(), count.data_ptr(),
                _stream_ptr(stream))
    _check(rc, "ardiff_entropy_gate_noalloc")
    return mask, idx, count


class Head:
    """Owns an ardiff_head handle (device weights + scratch)."""

    def __init__(self, C: int, Dc: int, W: int, L: int, F: int, K_max: int, max_tokens: int,
                 weights: Dict[str, "object"]):
        import numpy as np
        L_ = lib()
        self.desc = HeadDesc(C=C, Dc=Dc, W=W, L=L, F=F, K_max=K_max, max_tokens=max_tokens)
        keep = {k: np.ascontiguousarray(weights[k]) for k in _WEIGHT_FIELDS}
        for k, a in keep.items():
            assert a.dtype == np.uint16, f"{k}: bf16 bit patterns (uint16) expected"
        hw = HeadHostWeights(**{k: keep[k].ctypes.data for k in _WEIGHT_FIELDS})
        h = ctypes.c_void_p()
        _check(L_.ardiff_head_create(ctypes.byref(self.desc), ctypes.byref(hw), ctypes.byref(h)),
               "ardiff_head_create")
        self._h = h

    def ardiff_head_sample(self, cond, noise, t_sched, idx, count, out, stream=None):
        """K = len(t_sched)-1 steps for the survivors idx[0..*count); writes rows of `out`."""
        import numpy as np
        import torch
        assert cond.is_cuda and cond.dtype == torch.bfloat16 and cond.is_contiguous()
        assert noise.is_cuda and noise.dtype == torch.float32 and noise.is_contiguous()
        assert out.is_cuda and out.dtype == torch.float32 and out.is_contiguous()
        assert idx.dtype == torch.int32 and count.dtype == torch.int32
        ts = np.ascontiguousarray(t_sched, dtype=np.float32)
        K = ts.shape[0] - 1
        with _on(cond.device):
            rc = lib().ardiff_head_sample(self._h, cond.data_ptr(), noise.data_ptr(), ts.ctypes.data, K,
                                          idx.data_ptr(), count.data_ptr(), out.data_ptr(),
                                          _stream_ptr(stream))
        _check(rc, "ardiff_head_sample")
        return out

    def ardiff_head_sample_coef(self, cond, noise, t_in, coef, idx, count, out, step_noise=None, stream=None):
        """K = len(t_in) head evaluations, each followed by x <- ax x + av v + an z_k.
        coef: [K, 3] (ax, av, an); step_noise: float32 CUDA tensor [K, n, C] or None."""
        import numpy as np
        import torch
        assert cond.is_cuda and cond.dtype == torch.bfloat16 and cond.is_contiguous()
        assert noise.is_cuda and noise.dtype == torch.float32 and noise.is_contiguous()
        assert out.is_cuda and out.dtype == torch.float32 and out.is_contiguous()
        ts = np.ascontiguousarray(t_in, dtype=np.float32)
        cf = np.ascontiguousarray(coef, dtype=np.float32)
        K = ts.shape[0]
        assert cf.shape == (K, 3)
        n = noise.shape[0]
        if step_noise is not None:
            assert step_noise.is_cuda and step_noise.dtype == torch.float32 and step_noise.is_contiguous()
            assert tuple(step_noise.shape) == (K, n, noise.shape[1])
        fn = lib().ardiff_head_sample_coef
        with _on(cond.device):
            rc = fn(self._h, cond.data_ptr(), noise.data_ptr(), ts.ctypes.data, K, cf.ctypes.data,
                    step_noise.data_ptr() if step_noise is not None else None, n, idx.data_ptr(), count.data_ptr(),
                    out.data_ptr(), _stream_ptr(stream))
        _check(rc, "ardiff_head_sample_coef")
        return out

    def status(self, stream=None) -> int:
        return int(lib().ardiff_head_status(self._h, _stream_ptr(stream)))

    def set_timing(self, on: bool):
        _check(lib().ardiff_head_set_timing(self._h, 1 if on else 0), "ardiff_head_set_timing")

    def last_kernel_ms(self) -> float:
        ms = ctypes.c_float(0.0)
        _check(lib().ardiff_head_last_kernel_ms(self._h, ctypes.byref(ms)), "ardiff_head_last_kernel_ms")
        return float(ms.value)

    def last_kernel_clock_mhz(self, stream=None) -> float:
        """SM clock the last head kernel ran at (cycles / wall time, stamped on the device)."""
        mhz = ctypes.c_double(0.0)
        fn = lib().ardiff_head_last_kernel_clock
        _check(fn(self._h, _stream_ptr(stream), ctypes.byref(mhz)), "ardiff_head_last_kernel_clock")
        return float(mhz.value)

    def set_cooperative(self, on: bool):
        fn = lib().ardiff_head_set_cooperative
        _check(fn(self._h, 1 if on else 0), "ardiff_head_set_cooperative")

    def few_limits(self, K: int):
        """(chain, clusters): the survivors up to which a call of K steps takes either schedule; above both it takes the tiles."""
        chain, clusters = ctypes.c_int32(0), ctypes.c_int32(0)
        _check(lib().ardiff_head_few_limits(self._h, K, ctypes.byref(chain), ctypes.byref(clusters)), "ardiff_head_few_limits")
        return int(chain.value), int(clusters.value)

    def inject_stall(self, token_tile: int, wait_limit_us: int):
        """Arms the bounded-wait self-test for the next sample call (see ardiff_head_inject_stall)."""
        fn = lib().ardiff_head_inject_stall
        _check(fn(self._h, token_tile, wait_limit_us), "ardiff_head_inject_stall")

    def inject_cluster_stall(self, cluster: int, wait_limit_us: int):
        """The same for a wait inside a cluster (see ardiff_head_inject_cluster_stall)."""
        _check(lib().ardiff_head_inject_cluster_stall(self._h, cluster, wait_limit_us), "ardiff_head_inject_cluster_stall")

    def close(self):
        if getattr(self, "_h", None) is not None and self._h:
            lib().ardiff_head_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Pipeline:
    """Host-buffer front end (ardiff_pipeline_*): device staging for up to max_n tokens.

    With slots >= 2 the overlapped calls (ardiff_pipeline_submit / _wait / _join) are available."""

    def __init__(self, head: Head, max_n: int, d: int, slots: int = 1):
        self.head = head
        self.d, self.Dc, self.C = d, head.desc.Dc, head.desc.C
        self.slots = slots
        self._counts = [ctypes.c_int32(0) for _ in range(slots)]
        p = ctypes.c_void_p()
        fn = lib().ardiff_pipeline_create_slots
        _check(fn(head._h, max_n, d, self.Dc, self.C, slots, ctypes.byref(p)), "ardiff_pipeline_create_slots")
        self._p = p

    def ardiff_pipeline_run_host(self, feat, cond, noise, tau, t_sched, out, mask, stream=None) -> int:
        """feat/cond: host bf16 tensors, noise/out: host f32, mask: host u8 (pinned or not).
        Returns the number of kept tokens. Synchronises the stream."""
        import numpy as np
        ts = np.ascontiguousarray(t_sched, dtype=np.float32)
        n = feat.shape[0]
        count = ctypes.c_int32(0)
        rc = lib().ardiff_pipeline_run_host(self._p, feat.data_ptr(), cond.data_ptr(), noise.data_ptr(), n,
                                            float(tau), ts.ctypes.data, ts.shape[0] - 1, out.data_ptr(),
                                            mask.data_ptr(), ctypes.addressof(count), _stream_ptr(stream))
        _check(rc, "ardiff_pipeline_run_host")
        return int(count.value)

    def ardiff_pipeline_submit(self, slot: int, feat, cond, noise, tau, t_sched, out, mask, stream=None) -> None:
        """Enqueue one batch on `slot` without waiting; the host tensors must stay alive (and should
        be pinned) until ardiff_pipeline_wait(slot)."""
        import numpy as np
        ts = np.ascontiguousarray(t_sched, dtype=np.float32)
        fn = lib().ardiff_pipeline_submit
        if not 0 <= slot < self.slots:
            raise ValueError("slot out of range")
        rc = fn(self._p, slot, feat.data_ptr(), cond.data_ptr(), noise.data_ptr(), feat.shape[0], float(tau),
                ts.ctypes.data, ts.shape[0] - 1, out.data_ptr(), mask.data_ptr(),
                ctypes.addressof(self._counts[slot]), _stream_ptr(stream))
        _check(rc, "ardiff_pipeline_submit")

    def ardiff_pipeline_wait(self, slot: int) -> int:
        """Block until the batch on `slot` has been copied out; returns its number of kept tokens."""
        fn = lib().ardiff_pipeline_wait
        _check(fn(self._p, slot), "ardiff_pipeline_wait")
        return int(self._counts[slot].value)

    def ardiff_pipeline_join(self, stream=None) -> None:
        """Make `stream` wait on the device for every batch submitted so far."""
        fn = lib().ardiff_pipeline_join
        _check(fn(self._p, _stream_ptr(stream)), "ardiff_pipeline_join")

    def close(self):
        if getattr(self, "_p", None) is not None and self._p:
            lib().ardiff_pipeline_destroy(self._p)
            self._p = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
