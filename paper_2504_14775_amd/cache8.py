"""ctypes binding of the operators over a KV cache held in 8 bits (include/gllm_cache8.h): checks of the tensors and argument
marshalling only.  Every tensor lies on the current GPU; what a call refuses raises GllmError."""
from __future__ import annotations

import ctypes as C
import math

import torch

from .binding import GLLM_OK, GllmError, load_library
from .branch import _check, _own_workspace, _refuse, _row_stride, _stream

EXPORTS = ["gllm_op_step_maps", "gllm_op_norm_rope_store8", "gllm_op_attention8", "gllm_op_attention8_workspace_bytes"]
PAGE = 16

_device = torch._C._cuda_getDevice if hasattr(torch._C, "_cuda_getDevice") else None
_ready = None


def _lib():
    global _ready
    if _ready is None:
        lib = load_library()
        i32, i64, vp, sz = C.c_int32, C.c_int64, C.c_void_p, C.c_size_t
        lib.gllm_op_step_maps.restype = i32
        lib.gllm_op_step_maps.argtypes = [vp, vp, i32, vp, i32, vp, i32, i64, i32, vp, vp, vp, vp, vp]
        lib.gllm_op_norm_rope_store8.restype = i32
        lib.gllm_op_norm_rope_store8.argtypes = [vp, i64, i32, vp, vp, C.c_double, vp, i32, vp, vp, i32, i32, i32, i32, vp, i64, vp, vp, vp, i64, vp]
        lib.gllm_op_attention8.restype = i32
        lib.gllm_op_attention8.argtypes = [vp, i64, vp, vp, vp, i64, vp, i32, vp, vp, i32, i32, i32, i32, i32, i32, i32, i32, C.c_float, vp, i64,
                                           vp, sz, vp]
        lib.gllm_op_attention8_workspace_bytes.restype = sz
        lib.gllm_op_attention8_workspace_bytes.argtypes = [i32, i32, i32, i32]
        _ready = lib
    return _ready


_BF16, _F32, _I32, _U8, _E4M3 = torch.bfloat16, torch.float32, torch.int32, torch.uint8, torch.float8_e4m3fn


# A call's tensors are checked by one expression first, which takes a microsecond less than a loop over them; where it does not hold, _check says what is
# wrong, or that nothing is (rows with strides).


def _pool_shape(call: str, k_pool, v_pool, scales):
    """(pages, KV heads, head size) of a layer's pools; codes are uint8 or float8_e4m3fn."""
    v = v_pool.shape
    pages, n_kv, d = v[:3] if len(v) == 4 and v[3] == PAGE else (0, 0, 0)
    if d == 0 or d % 16 != 0 or k_pool.shape != (pages, n_kv, 4, d // 16, 4, 16) or scales.shape != (pages, n_kv, 2):
        _refuse(f"{call}: pools of shapes {tuple(k_pool.shape)}, {tuple(v)} and {tuple(scales.shape)}")
    for t in (k_pool.dtype, v_pool.dtype):
        if t is not _U8 and t is not _E4M3:
            _refuse(f"{call}: codes are uint8 or float8_e4m3fn, got {t}")
    return pages, n_kv, d


def gllm_op_step_maps(new_tokens, cached_len, free_pages, block_tables, num_blocks: int, row_start, positions, slots, needed, stream=None) -> None:
    """new_tokens, cached_len: int32 [S]; free_pages: int32 [F]; block_tables: int32 [S, entries], extended; row_start: int32 [S+1],
    positions, slots: int32 [R], needed: int32 [2], written."""
    call = "gllm_op_step_maps"
    dev = new_tokens.get_device()
    if not (dev >= 0 and cached_len.get_device() == free_pages.get_device() == block_tables.get_device() == row_start.get_device() ==
            positions.get_device() == slots.get_device() == needed.get_device() == dev == _device() and
            new_tokens.dtype is cached_len.dtype is free_pages.dtype is block_tables.dtype is _I32 and
            row_start.dtype is positions.dtype is slots.dtype is needed.dtype is _I32 and
            new_tokens.is_contiguous() and cached_len.is_contiguous() and free_pages.is_contiguous() and block_tables.is_contiguous() and
            row_start.is_contiguous() and positions.is_contiguous() and slots.is_contiguous() and needed.is_contiguous()):
        _check(call, ((new_tokens, _I32), (cached_len, _I32), (free_pages, _I32), (block_tables, _I32), (row_start, _I32), (positions, _I32), (slots, _I32),
                      (needed, _I32)))
    seqs, rows = new_tokens.numel(), slots.numel()
    if free_pages.dim() != 1 or cached_len.numel() != seqs or block_tables.dim() != 2 or block_tables.shape[0] != seqs or \
            row_start.numel() != seqs + 1 or positions.numel() != rows or needed.numel() != 2:
        _refuse(f"{call}: shapes new_tokens {tuple(new_tokens.shape)}, cached_len {tuple(cached_len.shape)}, "
                f"free_pages {tuple(free_pages.shape)}, block_tables {tuple(block_tables.shape)}, "
                f"row_start {tuple(row_start.shape)}, positions {tuple(positions.shape)}, slots {tuple(slots.shape)}, needed {tuple(needed.shape)}")
    if (seqs | rows | free_pages.numel() | block_tables.shape[1]) >> 31:
        _refuse(f"{call}: {seqs} sequences, {rows} rows, {free_pages.numel()} pages or tables of {block_tables.shape[1]} entries")
    st = _lib().gllm_op_step_maps(new_tokens.data_ptr(), cached_len.data_ptr(), seqs, free_pages.data_ptr(), free_pages.numel(), block_tables.data_ptr(),
                                  block_tables.shape[1], num_blocks, rows, row_start.data_ptr(), positions.data_ptr(), slots.data_ptr(),
                                  needed.data_ptr(), _stream(stream, dev))
    if st != GLLM_OK:
        raise GllmError(st, call)


def gllm_op_norm_rope_store8(qkv, q_gain, k_gain, eps: float, rope, positions, slots, q_out, k_pool, v_pool, scales, stream=None) -> None:
    """qkv: fp32 or bf16 [R, (n_q+2*n_kv)*d]; q_gain, k_gain: bf16 [d] or None; rope: fp32 [max_position, d/2, 2]; positions, slots: int32 [R];
    q_out: bf16 [R, n_q*d]; k_pool: [pages, n_kv, 4, d/16, 4, 16] and v_pool: [pages, n_kv, d, 16], uint8 or float8_e4m3fn; scales: fp32
    [pages, n_kv, 2]."""
    call = "gllm_op_norm_rope_store8"
    pages, n_kv, d = _pool_shape(call, k_pool, v_pool, scales)
    if qkv.dtype is not _F32 and qkv.dtype is not _BF16:
        _refuse(f"{call}: rows are float32 or bfloat16, got {qkv.dtype}")
    dev = qkv.get_device()
    if not (dev >= 0 and rope.get_device() == positions.get_device() == slots.get_device() == q_out.get_device() == k_pool.get_device() ==
            v_pool.get_device() == scales.get_device() == dev == _device() and rope.dtype is scales.dtype is _F32 and
            positions.dtype is slots.dtype is _I32 and q_out.dtype is _BF16 and qkv.is_contiguous() and rope.is_contiguous() and
            positions.is_contiguous() and slots.is_contiguous() and q_out.is_contiguous() and k_pool.is_contiguous() and v_pool.is_contiguous() and
            scales.is_contiguous()):
        _check(call, ((qkv, qkv.dtype), (rope, _F32), (positions, _I32), (slots, _I32), (q_out, _BF16), (k_pool, k_pool.dtype), (v_pool, v_pool.dtype),
                      (scales, _F32)), rows_only=(qkv, q_out))
    for g in (q_gain, k_gain):
        if g is not None and not (g.get_device() == dev and g.dtype is _BF16 and g.is_contiguous() and g.numel() == d):
            _check(call, ((qkv, qkv.dtype), (g, _BF16)), rows_only=(qkv,))
            _refuse(f"{call}: a gain of shape {tuple(g.shape)} for heads of {d}")
    rows, table = slots.numel(), rope.shape
    width = q_out.shape[1] if q_out.dim() == 2 else 0
    if qkv.shape != (rows, width + 2 * n_kv * d) or q_out.shape != (rows, width) or width % d != 0 or positions.numel() != rows or \
            rope.dim() != 3 or table[1] != d // 2 or table[2] != 2:
        _refuse(f"{call}: shapes qkv {tuple(qkv.shape)}, q_out {tuple(q_out.shape)}, rope {tuple(table)}, positions {tuple(positions.shape)}, "
                f"slots {tuple(slots.shape)}, {n_kv} KV heads of {d}")
    st = _lib().gllm_op_norm_rope_store8(qkv.data_ptr(), _row_stride(qkv), 0 if qkv.dtype is _F32 else 1, None if q_gain is None else q_gain.data_ptr(),
                                         None if k_gain is None else k_gain.data_ptr(), eps, rope.data_ptr(), table[0], positions.data_ptr(),
                                         slots.data_ptr(), rows, width // d, n_kv, d, q_out.data_ptr(), _row_stride(q_out), k_pool.data_ptr(),
                                         v_pool.data_ptr(), scales.data_ptr(), pages, _stream(stream, dev))
    if st != GLLM_OK:
        raise GllmError(st, call)


def gllm_op_attention8_workspace_bytes(n_q_heads: int, n_kv_heads: int, head_dim: int, max_new: int) -> int:
    return int(_lib().gllm_op_attention8_workspace_bytes(n_q_heads, n_kv_heads, head_dim, max_new))


def gllm_op_attention8(q, k_pool, v_pool, scales, block_tables, cached_len, row_start, out, max_new: int, window: int = 0, sinks: int = 0, scale=None,
                       workspace=None, stream=None) -> None:
    """q, out: bf16 [R, n_q*d]; pools and scales as above; block_tables: int32 [S, entries]; cached_len: int32 [S]; row_start: int32 [S+1].
    scale: 1/sqrt(d) if not given; workspace: uint8, taken from torch's allocator if not given."""
    call = "gllm_op_attention8"
    pages, n_kv, d = _pool_shape(call, k_pool, v_pool, scales)
    dev = q.get_device()
    if not (dev >= 0 and out.get_device() == k_pool.get_device() == v_pool.get_device() == scales.get_device() == block_tables.get_device() ==
            cached_len.get_device() == row_start.get_device() == dev == _device() and q.dtype is out.dtype is _BF16 and scales.dtype is _F32 and
            block_tables.dtype is cached_len.dtype is row_start.dtype is _I32 and q.is_contiguous() and out.is_contiguous() and k_pool.is_contiguous() and
            v_pool.is_contiguous() and scales.is_contiguous() and block_tables.is_contiguous() and cached_len.is_contiguous() and
            row_start.is_contiguous()):
        _check(call, ((q, _BF16), (out, _BF16), (k_pool, k_pool.dtype), (v_pool, v_pool.dtype), (scales, _F32), (block_tables, _I32), (cached_len, _I32),
                      (row_start, _I32)), rows_only=(q, out))
    seqs = cached_len.numel()
    if q.dim() != 2 or q.shape[1] % d != 0 or out.shape != q.shape or block_tables.dim() != 2 or block_tables.shape[0] != seqs or row_start.numel() != seqs + 1:
        _refuse(f"{call}: shapes q {tuple(q.shape)}, out {tuple(out.shape)}, block_tables {tuple(block_tables.shape)}, cached_len {tuple(cached_len.shape)}, "
                f"row_start {tuple(row_start.shape)}")
    if (max_new | window | sinks | seqs | block_tables.shape[1]) >> 31:
        _refuse(f"{call}: max_new {max_new}, window {window}, sinks {sinks}, {seqs} sequences, tables of {block_tables.shape[1]} entries")
    n_q = q.shape[1] // d
    lib = _lib()
    if workspace is None:
        workspace = _own_workspace(call, int(lib.gllm_op_attention8_workspace_bytes(n_q, n_kv, d, max_new)), q, stream)
    elif workspace.get_device() != dev or workspace.dtype is not _U8 or not workspace.is_contiguous():
        _check(call, ((q, _BF16), (workspace, _U8)), rows_only=(q,))
    st = lib.gllm_op_attention8(q.data_ptr(), _row_stride(q), k_pool.data_ptr(), v_pool.data_ptr(), scales.data_ptr(), pages, block_tables.data_ptr(),
                                block_tables.shape[1], cached_len.data_ptr(), row_start.data_ptr(), seqs, q.shape[0], max_new, window, sinks, n_q, n_kv, d,
                                1.0 / math.sqrt(d) if scale is None else scale, out.data_ptr(), _row_stride(out), workspace.data_ptr(),
                                workspace.numel(), _stream(stream, dev))
    if st != GLLM_OK:
        raise GllmError(st, call)
