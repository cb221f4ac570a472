"""Python view of include/toploc_model.h: same names, argument marshalling only.

The operators of the passes that produce the activations a proof commits to.  torch is used for
device memory and streams.  Wrong arguments raise ToplocError before anything is enqueued; what
only the device can see comes back in status tensors (TOPLOC_SEQ_*).  What a call allocates (outputs
that are not given, its workspace) is memory of the stream it runs on.
"""
import ctypes
import struct

import torch

from . import binding
from .binding import TOPLOC_DTYPE_BF16, TOPLOC_DTYPE_FP32, ToplocError, _bytes_of, _empty

__all__ = [
    "TOPLOC_SEQ_OK", "TOPLOC_SEQ_BAD_LENGTH", "TOPLOC_SEQ_NO_PAGES", "TOPLOC_SEQ_TABLE_FULL", "TOPLOC_SEQ_BATCH_FULL",
    "TOPLOC_SEQ_BAD_PAGE", "TOPLOC_SEQ_WAIT_EXPIRED", "TOPLOC_SEQ_BAD_PARENT", "TOPLOC_SEQ_IN_USE", "TOPLOC_SEQ_NO_ROOM",
    "TOPLOC_NORM_OUT_SAME", "TOPLOC_NORM_OUT_E4M3", "TOPLOC_ROTARY_HALVES", "TOPLOC_ROTARY_NEIGHBOURS",
    "TOPLOC_MAX_ALTERNATIVES", "ToplocKvLayout", "ToplocAttentionLayout", "ToplocNormLayout", "ToplocPoolLayout",
    "ToplocRotaryLayout", "ToplocLogprobLayout", "toploc_sequence_status_string",
    "toploc_plan_pages", "toploc_cache_write", "toploc_attention_workspace_bytes",
    "toploc_attention_paged", "toploc_attention_prompt", "toploc_rmsnorm_residual",
    "toploc_fork_pages", "toploc_release_pages", "toploc_compact_pages", "toploc_copy_pages",
    "toploc_norm_rotary_prompt", "toploc_norm_rotary_paged", "toploc_token_logprobs",
]

TOPLOC_SEQ_OK = 0
TOPLOC_SEQ_BAD_LENGTH = 1
TOPLOC_SEQ_NO_PAGES = 2
TOPLOC_SEQ_TABLE_FULL = 3
TOPLOC_SEQ_BATCH_FULL = 4
TOPLOC_SEQ_BAD_PAGE = 5
TOPLOC_SEQ_WAIT_EXPIRED = 6
TOPLOC_SEQ_BAD_PARENT = 7
TOPLOC_SEQ_IN_USE = 8
TOPLOC_SEQ_NO_ROOM = 9
TOPLOC_NORM_OUT_SAME = 0
TOPLOC_NORM_OUT_E4M3 = 1
TOPLOC_ROTARY_HALVES = 0
TOPLOC_ROTARY_NEIGHBOURS = 1
TOPLOC_MAX_ALTERNATIVES = 32

_DTYPES = {torch.bfloat16: TOPLOC_DTYPE_BF16, torch.float32: TOPLOC_DTYPE_FP32}
_i32, _i64, _vp = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p


class ToplocKvLayout(ctypes.Structure):
    _fields_ = [("page_size", _i32), ("num_pages", _i32), ("max_pages", _i32), ("reserved", _i32),
                ("table_stride", _i64), ("k_page_stride", _i64), ("k_token_stride", _i64), ("k_head_stride", _i64),
                ("v_page_stride", _i64), ("v_token_stride", _i64), ("v_head_stride", _i64)]


class ToplocAttentionLayout(ctypes.Structure):
    _fields_ = [("dtype", _i32), ("head_dim", _i32), ("q_heads", _i32), ("kv_heads", _i32), ("num_seqs", _i32),
                ("max_new_tokens", _i32), ("total_tokens", _i64), ("scale", ctypes.c_float), ("wait_tries", _i32),
                ("q_token_stride", _i64), ("q_head_stride", _i64), ("out_token_stride", _i64),
                ("out_head_stride", _i64)]


class ToplocNormLayout(ctypes.Structure):
    _fields_ = [("dtype", _i32), ("out_kind", _i32), ("group", _i32), ("hidden", _i32), ("rows", _i64),
                ("x_stride", _i64), ("residual_stride", _i64), ("residual_out_stride", _i64), ("y_stride", _i64)]


class ToplocPoolLayout(ctypes.Structure):
    _fields_ = [("dtype", _i32), ("num_pages", _i32), ("page_size", _i32), ("kv_heads", _i32), ("head_dim", _i32),
                ("num_caches", _i32), ("page_stride", _i64), ("token_stride", _i64), ("head_stride", _i64)]


class ToplocRotaryLayout(ctypes.Structure):
    _fields_ = [("dtype", _i32), ("head_dim", _i32), ("q_heads", _i32), ("kv_heads", _i32), ("rotary_dim", _i32),
                ("pairing", _i32), ("num_tokens", _i64), ("eps", ctypes.c_float), ("reserved", _i32),
                ("q_token_stride", _i64), ("q_head_stride", _i64), ("k_token_stride", _i64), ("k_head_stride", _i64),
                ("v_token_stride", _i64), ("v_head_stride", _i64), ("q_out_token_stride", _i64),
                ("q_out_head_stride", _i64), ("k_out_token_stride", _i64), ("k_out_head_stride", _i64)]


class ToplocLogprobLayout(ctypes.Structure):
    _fields_ = [("dtype", _i32), ("vocab", _i32), ("top", _i32), ("reserved", _i32), ("rows", _i64),
                ("row_stride", _i64)]


# The structures as the wrappers pass them: their bytes (packing is several times as fast as ctypes fields, and a
# decode step's call is short)
_KV, _ATTENTION, _NORM = struct.Struct("=4i7q"), struct.Struct("=6iqfi4q"), struct.Struct("=4i5q")
_POOL, _ROTARY, _LOGPROB = struct.Struct("=6i3q"), struct.Struct("=6iqfi10q"), struct.Struct("=4i2q")

_LIB = None


def _library():
    """The library with this header's entry points declared."""
    global _LIB
    if _LIB is None:
        lib = binding.load_library()
        kv_p = att_p = norm_p = _vp  # a structure by reference, or its bytes
        lib.toploc_sequence_status_string.restype = ctypes.c_char_p
        lib.toploc_sequence_status_string.argtypes = [ctypes.c_int]
        lib.toploc_plan_pages.restype = ctypes.c_int
        lib.toploc_plan_pages.argtypes = [_vp, _vp, _i32, _vp, _i32, _vp, _i32, _vp, _i32, _i64, _vp, _vp, _vp, _vp,
                                          _i64, _vp, _vp, _vp]
        lib.toploc_cache_write.restype = ctypes.c_int
        lib.toploc_cache_write.argtypes = [_vp, _vp, _i64, _i64, _i64, _i64, _vp, _i64, _i32, _i32, _i32, _vp, _vp,
                                           kv_p, _vp]
        lib.toploc_attention_workspace_bytes.restype = ctypes.c_size_t
        lib.toploc_attention_workspace_bytes.argtypes = [att_p, kv_p]
        lib.toploc_attention_paged.restype = ctypes.c_int
        lib.toploc_attention_paged.argtypes = [_vp, _vp, _vp, att_p, kv_p, _vp, _vp, _vp, _vp, _vp, _vp, _vp,
                                               ctypes.c_size_t, _vp]
        lib.toploc_attention_prompt.restype = ctypes.c_int
        lib.toploc_attention_prompt.argtypes = [_vp, _vp, _vp, att_p, kv_p, _vp, _vp, _vp, _vp, _vp, ctypes.c_size_t,
                                                _vp]
        lib.toploc_rmsnorm_residual.restype = ctypes.c_int
        lib.toploc_rmsnorm_residual.argtypes = [_vp, _vp, _vp, ctypes.c_float, norm_p, _vp,
                                                _vp, _vp, _vp]
        lib.toploc_fork_pages.restype = ctypes.c_int
        lib.toploc_fork_pages.argtypes = [_vp, _vp, _i32, _vp, _i32, _vp, _i32, _vp, _i32, _vp, _i32, _i64, _vp, _vp,
                                          _vp, _vp, _vp, _vp, _vp, _vp]
        lib.toploc_release_pages.restype = ctypes.c_int
        lib.toploc_release_pages.argtypes = [_vp, _vp, _i32, _vp, _i32, _i64, _vp, _i32, _i32, _vp, _i32, _vp, _vp, _vp,
                                             _vp, _vp, _vp]
        lib.toploc_compact_pages.restype = ctypes.c_int
        lib.toploc_compact_pages.argtypes = [_vp, _i32, _vp, _i32, _i64, _vp, _i32, _i32, _vp, _i64, _vp, _vp, _i32,
                                             _vp, _vp, _vp, _vp, _vp, _vp]
        lib.toploc_copy_pages.restype = ctypes.c_int
        lib.toploc_copy_pages.argtypes = [_vp, _vp, _vp, _vp, _vp, _i32, _vp]
        lib.toploc_norm_rotary_prompt.restype = ctypes.c_int
        lib.toploc_norm_rotary_prompt.argtypes = [_vp] * 10
        lib.toploc_norm_rotary_paged.restype = ctypes.c_int
        lib.toploc_norm_rotary_paged.argtypes = [_vp] * 14
        lib.toploc_token_logprobs.restype = ctypes.c_int
        lib.toploc_token_logprobs.argtypes = [_vp] * 8
        _LIB = lib
    return _LIB


def toploc_sequence_status_string(code):
    return _library().toploc_sequence_status_string(int(code)).decode()


def _need(condition, what):
    if not condition:
        raise ToplocError(what)


def _device(name, *tensors):
    """All tensors (None: absent) on one CUDA device, which is returned."""
    index = tensors[0].get_device()
    for t in tensors:
        if t is not None and t.get_device() != index:
            index = -1
    if index < 0:  # the CPU's number
        raise ToplocError("%s needs CUDA tensors of one device" % name)
    return tensors[0].device


def _vector(t, dtype, length, what):
    if t.dtype is not dtype or t.shape != (length,) or not t.is_contiguous():
        raise ToplocError("%s must be a contiguous %s tensor of %d entries" % (what, dtype, length))


def _ptr(t):
    return None if t is None else t.data_ptr()


def _pack(layout, *fields):
    try:
        return layout.pack(*fields)
    except struct.error as e:  # a number that does not fit its field
        raise ToplocError("a size, bound or stride is out of range: %s" % e)


def _call(fn, name, dev, stream, *args):
    """fn(*args, stream) with `dev` current; raises on a non-zero return code."""
    index = dev.index
    raw = torch._C._cuda_getCurrentRawStream(index) if stream is None else stream.cuda_stream
    if index == torch._C._cuda_getDevice():
        rc = fn(*args, raw)
    else:
        with torch.cuda.device(dev):
            rc = fn(*args, raw)
    if rc != 0:
        raise ToplocError("%s failed: %s (%d)" % (name, binding.toploc_error_string(rc), rc))


def toploc_plan_pages(cached_lens, new_lens, free_pages, first_free, block_table, page_size, seq_offsets, kv_lens,
                      slots, positions, next_free, status, stream=None):
    """Plans one step of a paged cache (see the header).  int32 CUDA tensors cached_lens, new_lens, kv_lens [n],
    free_pages [any], first_free, next_free [1], block_table [n, max_pages], seq_offsets [n + 1], positions
    [max_tokens]; slots int64 [max_tokens], status uint8 [n].  The last six are written, and the block table."""
    dev = _device("toploc_plan_pages", cached_lens, new_lens, free_pages, first_free, block_table, seq_offsets, kv_lens,
                  slots, positions, next_free, status)
    n, tokens, i32 = cached_lens.numel(), slots.numel(), torch.int32
    if not (cached_lens.dtype is new_lens.dtype is free_pages.dtype is first_free.dtype is seq_offsets.dtype is
            kv_lens.dtype is positions.dtype is next_free.dtype is i32 and
            new_lens.shape == kv_lens.shape == status.shape == (n,) and seq_offsets.shape == (n + 1,) and
            positions.shape == (tokens,) and first_free.shape == next_free.shape == (1,) and free_pages.dim() == 1 and
            slots.dtype is torch.int64 and status.dtype is torch.uint8):
        raise ToplocError("toploc_plan_pages: int32 cached_lens, new_lens, kv_lens [n], free_pages, first_free and "
                          "next_free [1], seq_offsets [n + 1], positions [tokens]; int64 slots [tokens], uint8 status [n]")
    for t in (cached_lens, new_lens, free_pages, seq_offsets, kv_lens, slots, positions, status):
        _need(t.is_contiguous(), "toploc_plan_pages needs contiguous vectors")
    _need(block_table.dtype == i32 and block_table.dim() == 2 and block_table.shape[0] == n and
          (block_table.stride(1) == 1 or block_table.shape[1] <= 1 or n == 0), "block_table must be int32 [n, max_pages]")
    width = block_table.shape[1]
    _call(_library().toploc_plan_pages, "toploc_plan_pages", dev, stream, _ptr(cached_lens), _ptr(new_lens), n,
          _ptr(free_pages), free_pages.shape[0], _ptr(first_free), page_size, _ptr(block_table), width,
          block_table.stride(0) if n > 1 else width, _ptr(seq_offsets), _ptr(kv_lens), _ptr(slots), _ptr(positions),
          tokens, _ptr(next_free), _ptr(status))


def _cache_layout(k_cache, v_cache, block_table=None):
    """Layout of a cache [num_pages, page_size, kv_heads, head_dim]; a permuted view gives any order."""
    shape, k_strides, v_strides = k_cache.shape, k_cache.stride(), v_cache.stride()
    _need(len(shape) == 4 and v_cache.shape == shape and k_cache.dtype is v_cache.dtype and
          k_strides[3] == 1 and v_strides[3] == 1,
          "the caches must be [pages, page_size, kv_heads, head_dim] of one type, the last dimension contiguous")
    width = 0 if block_table is None else block_table.shape[1]
    stride = 0 if block_table is None else block_table.stride(0) if block_table.shape[0] > 1 else width
    (pages, page, _, _), (kp, kt, kh, _), (vp, vt, vh, _) = shape, k_strides, v_strides
    return _pack(_KV, page, pages, width, 0, stride, kp, kt, kh, vp, vt, vh)


def toploc_cache_write(k, v, slots, k_cache, v_cache, stream=None):
    """Writes k, v [num_tokens, kv_heads, head_dim] to their slots (int64 [num_tokens], negative: skipped) of the
    caches [num_pages, page_size, kv_heads, head_dim]."""
    dev = _device("toploc_cache_write", k, v, slots, k_cache, v_cache)
    kv = _cache_layout(k_cache, v_cache)
    _need(k.dim() == 3 and k.shape == v.shape and k.dtype == v.dtype == k_cache.dtype and k.stride(2) == 1 and
          v.stride(2) == 1 and k.shape[1:] == k_cache.shape[2:],
          "k and v must be [tokens, kv_heads, head_dim] of the cache's type, the last dimension contiguous")
    _need(k.dtype in _DTYPES, "keys and values must be bfloat16 or float32")
    _vector(slots, torch.int64, k.shape[0], "slots")
    _call(_library().toploc_cache_write, "toploc_cache_write", dev, stream, _ptr(k), _ptr(v), k.stride(0), k.stride(1),
          v.stride(0), v.stride(1), _ptr(slots), k.shape[0], _DTYPES[k.dtype], k.shape[1], k.shape[2], _ptr(k_cache),
          _ptr(v_cache), kv)


def _attention_layout(q, kv_heads, num_seqs, max_new_tokens, scale, out, lse):
    _need(q.dim() == 3 and q.stride(2) == 1, "q must be [tokens, q_heads, head_dim], the last dimension contiguous")
    _need(q.dtype in _DTYPES, "attention takes bfloat16 or float32 tensors")
    tokens, heads, dim = q.shape
    _need(out.shape == q.shape and out.dtype == q.dtype and out.stride(2) == 1, "out must have q's shape and type")
    _need(lse is None or (lse.dtype == torch.float32 and lse.shape == q.shape[:2] and lse.is_contiguous()),
          "lse must be a contiguous float32 [tokens, q_heads]")
    (qt, qh, _), (ot, oh, _) = q.stride(), out.stride()
    return _pack(_ATTENTION, _DTYPES[q.dtype], dim, heads, kv_heads, num_seqs, max_new_tokens, tokens,
                 dim ** -0.5 if scale is None else scale, 0, qt, qh, ot, oh)


def _attention_workspace(lib, lay, kv, workspace, dev, stream):
    if workspace is None:
        need = lib.toploc_attention_workspace_bytes(lay, kv)
        if need == 0:
            return None, 0
        workspace = _empty((need,), torch.uint8, dev, stream, hidden=True)
    return workspace, _bytes_of(workspace)


def toploc_attention_workspace_bytes(q, k_cache, v_cache, block_table, max_new_tokens):
    """Bytes of workspace toploc_attention_paged needs for these tensors (0: none)."""
    lay = _attention_layout(q, k_cache.shape[2], block_table.shape[0], max_new_tokens, None, q, None)
    kv = _cache_layout(k_cache, v_cache, block_table)
    return int(_library().toploc_attention_workspace_bytes(lay, kv))


def toploc_attention_paged(q, k_cache, v_cache, block_table, seq_offsets, kv_lens, max_new_tokens, scale=None,
                           out=None, lse=None, want_lse=False, status=None, workspace=None, stream=None):
    """Causal attention of packed new tokens q [tokens, q_heads, head_dim] over the caches [num_pages, page_size,
    kv_heads, head_dim] that already hold them.  block_table int32 [n, max_pages], seq_offsets int32 [n + 1],
    kv_lens int32 [n]; max_new_tokens bounds a sequence's new tokens; scale: 1 / sqrt(head_dim) by default; status:
    uint8 [n], set where a sequence is not as promised (zeroed by the caller; one tensor may collect many calls).
    Without it lengths over their bounds and pages outside the cache go unnoticed, and a wait inside the kernel that
    ran out shows only as NaN rows.  Returns (out, lse or None)."""
    if out is None:
        out = _empty(q.shape, q.dtype, q.device, stream)
    if lse is None and want_lse:
        lse = _empty(q.shape[:2], torch.float32, q.device, stream)
    dev = _device("toploc_attention_paged", q, k_cache, v_cache, block_table, seq_offsets, kv_lens, out, lse, status,
                  workspace)
    n = kv_lens.shape[0]
    _vector(seq_offsets, torch.int32, n + 1, "seq_offsets")
    _vector(kv_lens, torch.int32, n, "kv_lens")
    _need(block_table.dtype == torch.int32 and block_table.dim() == 2 and block_table.shape[0] == n and
          (block_table.stride(1) == 1 or block_table.shape[1] <= 1 or n == 0), "block_table must be int32 [n, max_pages]")
    if status is not None:
        _vector(status, torch.uint8, n, "status")
    lay = _attention_layout(q, k_cache.shape[2], n, max_new_tokens, scale, out, lse)
    kv = _cache_layout(k_cache, v_cache, block_table)
    _need(k_cache.dtype == q.dtype and k_cache.shape[3] == q.shape[2], "the caches must have q's type and head_dim")
    lib = _library()
    workspace, size = _attention_workspace(lib, lay, kv, workspace, dev, stream)
    _call(lib.toploc_attention_paged, "toploc_attention_paged", dev, stream, _ptr(q), _ptr(k_cache), _ptr(v_cache),
          lay, kv, _ptr(block_table), _ptr(seq_offsets), _ptr(kv_lens), _ptr(out), _ptr(lse), _ptr(status),
          _ptr(workspace), size)
    return out, lse


def toploc_attention_prompt(q, k, v, seq_offsets, max_tokens, scale=None, out=None, lse=None, want_lse=False,
                            status=None, workspace=None, stream=None):
    """Causal attention over packed prompts: q [tokens, q_heads, head_dim], k and v [tokens, kv_heads, head_dim]
    (views of one tensor are fine), seq_offsets int32 [n + 1], max_tokens bounds a sequence's length; status as for
    toploc_attention_paged.  Returns (out, lse or None)."""
    if out is None:
        out = _empty(q.shape, q.dtype, q.device, stream)
    if lse is None and want_lse:
        lse = _empty(q.shape[:2], torch.float32, q.device, stream)
    dev = _device("toploc_attention_prompt", q, k, v, seq_offsets, out, lse, status, workspace)
    n = seq_offsets.shape[0] - 1
    _need(n >= 0, "seq_offsets must have num_seqs + 1 entries")
    _vector(seq_offsets, torch.int32, n + 1, "seq_offsets")
    if status is not None:
        _vector(status, torch.uint8, n, "status")
    _need(k.dim() == 3 and k.shape == v.shape and k.dtype == v.dtype == q.dtype and k.stride(2) == 1 and
          v.stride(2) == 1 and k.shape[0] == q.shape[0] and k.shape[2] == q.shape[2],
          "k and v must be [tokens, kv_heads, head_dim] of q's type, the last dimension contiguous")
    lay = _attention_layout(q, k.shape[1], n, max_tokens, scale, out, lse)
    kv = _pack(_KV, 0, 0, 0, 0, 0, 0, k.stride(0), k.stride(1), 0, v.stride(0), v.stride(1))
    lib = _library()
    workspace, size = _attention_workspace(lib, lay, kv, workspace, dev, stream)
    _call(lib.toploc_attention_prompt, "toploc_attention_prompt", dev, stream, _ptr(q), _ptr(k), _ptr(v), lay, kv,
          _ptr(seq_offsets), _ptr(out), _ptr(lse), _ptr(status), _ptr(workspace), size)
    return out, lse


def toploc_rmsnorm_residual(x, residual, weight, eps, residual_out=None, y=None, scales=None, group=0, quantize=None,
                            stream=None):
    """h = x + residual (None: h = x), y = h * rsqrt(mean(h^2) + eps) * weight; x, residual, residual_out
    [rows, hidden], weight [hidden], bfloat16 or float32.  y of x's type, or float8_e4m3fn with fp32 scales
    [rows, ceil(hidden / group)] (group 0: one per row); quantize: which of the two to allocate where y is None.
    residual_out may be residual itself; it is allocated where a residual is given and it is None.  Returns
    (y, residual_out, scales or None)."""
    _need(x.dtype in _DTYPES and x.dim() == 2 and x.stride(1) == 1, "x must be bfloat16 or float32 [rows, hidden]")
    rows, hidden = x.shape
    if y is None:
        y = _empty((rows, hidden), torch.float8_e4m3fn if quantize else x.dtype, x.device, stream)
    quant = y.dtype == torch.float8_e4m3fn
    _need(group >= 0, "group must not be negative")
    if quant and scales is None:
        scales = _empty((rows, 1 if group == 0 else -(-hidden // group)), torch.float32, x.device, stream)
    if residual is not None and residual_out is None:
        residual_out = _empty((rows, hidden), x.dtype, x.device, stream)
    dev = _device("toploc_rmsnorm_residual", x, residual, weight, residual_out, y, scales)
    strides = []
    for t, what in ((x, "x"), (residual, "residual"), (residual_out, "residual_out")):
        _need(t is None or (t.shape == x.shape and t.dtype == x.dtype and t.stride(1) == 1),
              "%s must have x's shape and type, rows contiguous" % what)
        strides.append(hidden if t is None or rows <= 1 else t.stride(0))
    _need(y.shape == x.shape and y.stride(1) == 1 and (quant or y.dtype == x.dtype),
          "y must have x's shape, and its type or float8_e4m3fn")
    _need(weight.shape == (hidden,) and weight.dtype == x.dtype and weight.is_contiguous(), "weight must be [hidden]")
    if quant:
        _need(scales.dtype == torch.float32 and scales.is_contiguous() and
              scales.shape == (rows, 1 if group == 0 else -(-hidden // group)),
              "scales must be contiguous float32 [rows, groups]")
    lay = _pack(_NORM, _DTYPES[x.dtype], TOPLOC_NORM_OUT_E4M3 if quant else TOPLOC_NORM_OUT_SAME, group, hidden, rows,
                strides[0], strides[1], strides[2], y.stride(0) if rows > 1 else hidden)
    _call(_library().toploc_rmsnorm_residual, "toploc_rmsnorm_residual", dev, stream, _ptr(x), _ptr(residual),
          _ptr(weight), eps, lay, _ptr(residual_out), _ptr(y), _ptr(scales) if quant else None)
    return y, residual_out, scales if quant else None


_PAIRINGS = {"halves": TOPLOC_ROTARY_HALVES, "neighbours": TOPLOC_ROTARY_NEIGHBOURS}


def _rotary_layout(q, k, v, positions, inv_freq, q_weight, k_weight, eps, pairing, q_out, k_out):
    dtype, q_shape, k_shape = q.dtype, q.shape, k.shape
    (tokens, heads, dim), (k_tokens, kv_heads, k_dim), pairs = q_shape, k_shape, inv_freq.numel()
    (qt, qh, q1), (kt, kh, k1), (ot, oh, o1) = q.stride(), k.stride(), q_out.stride()
    (vt, vh, v1), (pt, ph, p1) = (0, 0, 1) if v is None else v.stride(), (0, 0, 1) if k_out is None else k_out.stride()
    if not (dtype in _DTYPES and dtype is k.dtype is q_out.dtype and k_tokens == tokens and k_dim == dim and
            q_out.shape == q_shape and q1 == k1 == o1 == v1 == p1 == 1 and
            (v is None or (v.shape == k_shape and v.dtype is dtype)) and
            (k_out is None or (k_out.shape == k_shape and k_out.dtype is dtype))):
        raise ToplocError("queries and their output must be [tokens, q_heads, head_dim], keys, values and the keys' output "
                          "[tokens, kv_heads, head_dim], all bfloat16 or all float32, the last dimension contiguous")
    if not (positions.dtype is torch.int32 and positions.numel() == tokens and positions.is_contiguous() and
            inv_freq.dtype is torch.float32 and inv_freq.is_contiguous() and 2 * pairs <= dim):
        raise ToplocError("positions must be a contiguous int32 vector of %d entries, inv_freq a contiguous float32 vector of "
                          "at most head_dim / 2" % tokens)
    for weight in (q_weight, k_weight):
        if weight is not None and (weight.dtype is not dtype or weight.numel() != dim or not weight.is_contiguous()):
            raise ToplocError("a norm's weight must be [head_dim] of q's type")
    if pairing not in _PAIRINGS:
        raise ToplocError("pairing must be 'halves' or 'neighbours'")
    return _pack(_ROTARY, _DTYPES[dtype], dim, heads, kv_heads, 2 * pairs, _PAIRINGS[pairing], tokens, eps, 0, qt, qh, kt,
                 kh, vt, vh, ot, oh, pt, ph)


_DIMENSIONS = "%s takes queries, keys and values of three dimensions"


def toploc_norm_rotary_prompt(q, k, positions, inv_freq, q_weight=None, k_weight=None, eps=1e-6, pairing="halves",
                              q_out=None, k_out=None, stream=None):
    """RMS norm of every head of q [tokens, q_heads, head_dim] and k [tokens, kv_heads, head_dim] (a weight that is None:
    no norm of that one) and the rotation by position: positions int32 [tokens], inv_freq float32 [pairs]; the first
    2 * pairs channels of a head turn, channel c with c + pairs ("halves") or 2c with 2c + 1 ("neighbours").  q_out may be
    q, k_out may be k.  Returns (q_out, k_out)."""
    name = "toploc_norm_rotary_prompt"
    if q_out is None:
        q_out = _empty(q.shape, q.dtype, q.device, stream)
    if k_out is None:
        k_out = _empty(k.shape, k.dtype, k.device, stream)
    dev = _device(name, q, k, positions, inv_freq, q_weight, k_weight, q_out, k_out)
    if not q.dim() == k.dim() == q_out.dim() == k_out.dim() == 3:
        raise ToplocError(_DIMENSIONS % name)
    lay = _rotary_layout(q, k, None, positions, inv_freq, q_weight, k_weight, eps, pairing, q_out, k_out)
    _call(_library().toploc_norm_rotary_prompt, name, dev, stream, _ptr(q), _ptr(k),
          _ptr(positions), _ptr(inv_freq), _ptr(q_weight), _ptr(k_weight), lay, _ptr(q_out), _ptr(k_out))
    return q_out, k_out


def toploc_norm_rotary_paged(q, k, v, positions, slots, inv_freq, k_cache, v_cache, q_weight=None, k_weight=None,
                             eps=1e-6, pairing="halves", q_out=None, stream=None):
    """toploc_norm_rotary_prompt with the keys' result and the values v [tokens, kv_heads, head_dim] written straight to
    their slots (int64 [tokens], negative: skipped) of the caches [num_pages, page_size, kv_heads, head_dim].  Returns
    q_out."""
    name = "toploc_norm_rotary_paged"
    if q_out is None:
        q_out = _empty(q.shape, q.dtype, q.device, stream)
    dev = _device(name, q, k, v, positions, slots, inv_freq, k_cache, v_cache, q_weight, k_weight, q_out)
    if not q.dim() == k.dim() == v.dim() == q_out.dim() == 3:
        raise ToplocError(_DIMENSIONS % name)
    lay = _rotary_layout(q, k, v, positions, inv_freq, q_weight, k_weight, eps, pairing, q_out, None)
    kv = _cache_layout(k_cache, v_cache)
    (_, _, heads, dim), (tokens, kv_heads, head_dim) = k_cache.shape, k.shape
    if not (k_cache.dtype is q.dtype and heads == kv_heads and dim == head_dim and slots.dtype is torch.int64 and
            slots.numel() == tokens and slots.is_contiguous()):
        raise ToplocError("the caches must have k's type, heads and head_dim, slots must be a contiguous int64 vector of "
                          "as many entries as there are tokens")
    _call(_library().toploc_norm_rotary_paged, name, dev, stream, q.data_ptr(), k.data_ptr(), v.data_ptr(),
          positions.data_ptr(), slots.data_ptr(), inv_freq.data_ptr(), _ptr(q_weight), _ptr(k_weight), lay,
          q_out.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), kv)
    return q_out


def toploc_token_logprobs(logits, tokens=None, top=0, want_entropy=False, logprobs=None, entropy=None, top_ids=None,
                          top_logprobs=None, stream=None):
    """Of every row of logits [rows, vocab] (bfloat16 or float32): the log probability of its token (int64 [rows]; None:
    none), the entropy (where wanted, or a tensor is given), and the `top` likeliest tokens with their log probabilities,
    in order (equal logits by index).  Returns (logprobs [rows] or None, entropy [rows] or None, top_ids int64 [rows, top]
    or None, top_logprobs [rows, top] or None)."""
    _need(logits.dtype in _DTYPES and logits.dim() == 2 and (logits.stride(1) == 1 or logits.shape[1] == 1),
          "logits must be bfloat16 or float32 [rows, vocab]")
    _need(top >= 0, "top must not be negative")
    (rows, vocab), dev, fp32 = logits.shape, logits.device, torch.float32
    if tokens is None:
        _need(logprobs is None, "logprobs need tokens")
    elif logprobs is None:
        logprobs = _empty((rows,), fp32, dev, stream)
    if entropy is None and want_entropy:
        entropy = _empty((rows,), fp32, dev, stream)
    if top == 0:
        _need(top_ids is None and top_logprobs is None, "alternatives with top 0")
    else:
        if top_ids is None:
            top_ids = _empty((rows, top), torch.int64, dev, stream)
        if top_logprobs is None:
            top_logprobs = _empty((rows, top), fp32, dev, stream)
        _need(top_ids.dtype is torch.int64 and top_logprobs.dtype is fp32 and
              top_ids.shape == top_logprobs.shape == (rows, top) and top_ids.is_contiguous() and
              top_logprobs.is_contiguous(), "top_ids and top_logprobs must be contiguous int64 and float32 [rows, top]")
    dev = _device("toploc_token_logprobs", logits, tokens, logprobs, entropy, top_ids, top_logprobs)
    if tokens is not None:
        _vector(tokens, torch.int64, rows, "tokens")
        _vector(logprobs, fp32, rows, "logprobs")
    if entropy is not None:
        _vector(entropy, fp32, rows, "entropy")
    lay = _pack(_LOGPROB, _DTYPES[logits.dtype], vocab, top, 0, rows, logits.stride(0) if rows > 1 else vocab)
    _call(_library().toploc_token_logprobs, "toploc_token_logprobs", dev, stream, _ptr(logits), lay, _ptr(tokens),
          _ptr(logprobs), _ptr(entropy), _ptr(top_ids), _ptr(top_logprobs))
    return logprobs, entropy, top_ids, top_logprobs


def _table(t, n, what):
    """(columns, elements between rows) of a block table [n, max_pages]."""
    if t.dtype is torch.int32 and t.dim() == 2:
        (rows, width), (stride, one) = t.shape, t.stride()
        if rows == n and (one == 1 or width <= 1 or n == 0):
            return width, stride if n > 1 else width
    raise ToplocError("%s must be int32 [n, max_pages]" % what)


def toploc_fork_pages(parents, kv_lens, shares, free_pages, first_free, block_table, page_size, kv_lens_out, shares_out,
                      copy_from, copy_to, num_copies, next_free, status, stream=None):
    """Sequences with parents[i] >= 0 begin as copies of their parents (see the header): whole pages are shared, a page
    that is not full is copied, by toploc_copy_pages from the list that this leaves.  int32 CUDA tensors parents, kv_lens,
    kv_lens_out, copy_from, copy_to [n], shares, shares_out [num_pages], free_pages [any], first_free, num_copies,
    next_free [1], block_table [n, max_pages]; status uint8 [n].  The last seven are written, and the children's rows of
    the block table."""
    name, n = "toploc_fork_pages", parents.numel()
    dev = _device(name, parents, kv_lens, shares, free_pages, first_free, block_table, kv_lens_out, shares_out, copy_from,
                  copy_to, num_copies, next_free, status)
    pages, free = shares.numel(), free_pages.numel()
    i32 = torch.int32
    if not (parents.dtype is kv_lens.dtype is shares.dtype is free_pages.dtype is first_free.dtype is kv_lens_out.dtype is
            shares_out.dtype is copy_from.dtype is copy_to.dtype is num_copies.dtype is next_free.dtype is i32 and
            status.dtype is torch.uint8 and
            kv_lens.numel() == kv_lens_out.numel() == copy_from.numel() == copy_to.numel() == status.numel() == n and
            shares_out.numel() == pages and first_free.numel() == num_copies.numel() == next_free.numel() == 1 and
            parents.is_contiguous() and kv_lens.is_contiguous() and shares.is_contiguous() and
            free_pages.is_contiguous() and kv_lens_out.is_contiguous() and shares_out.is_contiguous() and
            copy_from.is_contiguous() and copy_to.is_contiguous() and status.is_contiguous()):
        raise ToplocError("toploc_fork_pages: contiguous int32 parents, kv_lens, kv_lens_out, copy_from, copy_to [n], shares, "
                          "shares_out [num_pages], free_pages, first_free, num_copies, next_free [1]; uint8 status [n]")
    width, stride = _table(block_table, n, "block_table")
    _call(_library().toploc_fork_pages, name, dev, stream, parents.data_ptr(), kv_lens.data_ptr(), n,
          shares.data_ptr(), pages, free_pages.data_ptr(), free, first_free.data_ptr(), page_size,
          block_table.data_ptr(), width, stride, kv_lens_out.data_ptr(), shares_out.data_ptr(), copy_from.data_ptr(),
          copy_to.data_ptr(), num_copies.data_ptr(), next_free.data_ptr(), status.data_ptr())


def toploc_release_pages(release, kv_lens, block_table, shares, page_size, free_pages, first_free, kv_lens_out,
                         shares_out, next_free, status, stream=None):
    """Sequences with release[i] != 0 (uint8 [n]) let go of their pages; those that nobody holds any longer go back to the
    free list, in front of its head (see the header).  int32 CUDA tensors kv_lens, kv_lens_out [n], shares, shares_out
    [num_pages], free_pages [any], first_free, next_free [1], block_table [n, max_pages]; status uint8 [n].  The last four
    are written, and the entries of free_pages in front of first_free."""
    name, n = "toploc_release_pages", kv_lens.numel()
    dev = _device(name, release, kv_lens, block_table, shares, free_pages, first_free, kv_lens_out, shares_out, next_free,
                  status)
    pages, free = shares.numel(), free_pages.numel()
    i32, u8 = torch.int32, torch.uint8
    if not (kv_lens.dtype is shares.dtype is free_pages.dtype is first_free.dtype is kv_lens_out.dtype is shares_out.dtype is
            next_free.dtype is i32 and release.dtype is status.dtype is u8 and
            release.numel() == kv_lens_out.numel() == status.numel() == n and shares_out.numel() == pages and
            first_free.numel() == next_free.numel() == 1 and release.is_contiguous() and kv_lens.is_contiguous() and
            shares.is_contiguous() and free_pages.is_contiguous() and kv_lens_out.is_contiguous() and
            shares_out.is_contiguous() and status.is_contiguous()):
        raise ToplocError("toploc_release_pages: contiguous int32 kv_lens, kv_lens_out [n], shares, shares_out [num_pages], "
                          "free_pages, first_free, next_free [1]; uint8 release, status [n]")
    width, stride = _table(block_table, n, "block_table")
    _call(_library().toploc_release_pages, name, dev, stream, release.data_ptr(), kv_lens.data_ptr(), n,
          block_table.data_ptr(), width, stride, shares.data_ptr(), pages, page_size, free_pages.data_ptr(), free,
          first_free.data_ptr(), kv_lens_out.data_ptr(), shares_out.data_ptr(), next_free.data_ptr(),
          status.data_ptr())


def toploc_compact_pages(kv_lens, block_table, shares, page_size, block_table_out, shares_out, free_pages_out, copy_from,
                         copy_to, num_copies, next_free, status, stream=None):
    """The pool's pages in use become its first ones (see the header); toploc_copy_pages moves their contents by the list
    that this leaves.  int32 CUDA tensors kv_lens [n], block_table, block_table_out [n, max_pages] (may be one tensor),
    shares, shares_out, copy_from, copy_to [num_pages], free_pages_out [num_pages or more], num_copies, next_free [1];
    status uint8 [n].  The last eight are written.  A call with one tensor for both tables is not to be repeated, or replayed,
    before shares holds what shares_out got."""
    name, n = "toploc_compact_pages", kv_lens.numel()
    dev = _device(name, kv_lens, block_table, shares, block_table_out, shares_out, free_pages_out, copy_from, copy_to,
                  num_copies, next_free, status)
    pages, free = shares.numel(), free_pages_out.numel()
    i32 = torch.int32
    if not (kv_lens.dtype is shares.dtype is shares_out.dtype is free_pages_out.dtype is copy_from.dtype is copy_to.dtype is
            num_copies.dtype is next_free.dtype is i32 and status.dtype is torch.uint8 and status.numel() == n and
            shares_out.numel() == copy_from.numel() == copy_to.numel() == pages and
            num_copies.numel() == next_free.numel() == 1 and kv_lens.is_contiguous() and shares.is_contiguous() and
            shares_out.is_contiguous() and free_pages_out.is_contiguous() and copy_from.is_contiguous() and
            copy_to.is_contiguous() and status.is_contiguous()):
        raise ToplocError("toploc_compact_pages: contiguous int32 kv_lens [n], shares, shares_out, copy_from, copy_to "
                          "[num_pages], free_pages_out, num_copies, next_free [1]; uint8 status [n]")
    width, stride = _table(block_table, n, "block_table")
    out_width, out_stride = _table(block_table_out, n, "block_table_out")
    _need(width == out_width, "block_table_out must have block_table's shape")
    _call(_library().toploc_compact_pages, name, dev, stream, kv_lens.data_ptr(), n, block_table.data_ptr(), width,
          stride, shares.data_ptr(), pages, page_size, block_table_out.data_ptr(), out_stride, shares_out.data_ptr(),
          free_pages_out.data_ptr(), free, copy_from.data_ptr(), copy_to.data_ptr(), num_copies.data_ptr(),
          next_free.data_ptr(), status.data_ptr())


def toploc_copy_pages(caches, copy_from, copy_to, num_copies, stream=None):
    """Copies page copy_from[c] to page copy_to[c], c < num_copies[0], inside every one of the caches, a list of CUDA
    tensors [num_pages, page_size, kv_heads, head_dim] of one type and layout (keys and values of all layers); copy_from,
    copy_to int32 [any], num_copies int32 [1]."""
    name = "toploc_copy_pages"
    if not caches:
        return
    one = caches[0]
    dev, shape, strides, dtype, most = _device(name, copy_from, copy_to, num_copies, one), one.shape, one.stride(), one.dtype, \
        copy_from.numel()
    index, pointers = dev.index, []
    if len(shape) != 4 or dtype not in _DTYPES or strides[3] != 1:
        raise ToplocError("caches must be bfloat16 or float32 [pages, page_size, kv_heads, head_dim], the last dimension "
                          "contiguous")
    for c in caches:
        if c.shape != shape or c.stride() != strides or c.dtype is not dtype or c.get_device() != index:
            raise ToplocError("caches must have one type and layout, and be on one device")
        pointers.append(c.data_ptr())
    i32 = torch.int32
    if not (copy_from.dtype is copy_to.dtype is num_copies.dtype is i32 and copy_from.shape == copy_to.shape == (most,) and
            num_copies.shape == (1,) and copy_from.is_contiguous() and copy_to.is_contiguous()):
        raise ToplocError("copy_from and copy_to must be contiguous int32 vectors of one length, num_copies int32 [1]")
    pages, tokens, heads, dim = shape
    lay = _pack(_POOL, _DTYPES[dtype], pages, tokens, heads, dim, len(pointers), strides[0], strides[1], strides[2])
    _call(_library().toploc_copy_pages, name, dev, stream, struct.pack("=%dQ" % len(pointers), *pointers), lay,
          copy_from.data_ptr(), copy_to.data_ptr(), num_copies.data_ptr(), most)
