"""ctypes binding of the operators for several continuations of one sequence (include/gllm_branch.h): checks of the tensors
and argument marshalling only.  Every tensor lies on the current GPU; what a call refuses raises GllmError."""
from __future__ import annotations

import ctypes as C
import math
from array import array

import numpy as np
import torch

from .binding import GLLM_OK, GllmError, _stream_ptr, load_library

EXPORTS = [
    "gllm_op_tree_attention", "gllm_op_tree_attention_workspace_bytes", "gllm_op_tree_commit", "gllm_op_beam_select",
    "gllm_op_beam_select_workspace_bytes", "gllm_op_copy_pages",
]
PAGE = 16
_INVALID, _BLOCK_RANGE = -1, -3

_ready = None


def _lib():
    global _ready
    if _ready is None:
        lib = load_library()
        i32, i64, vp, sz = C.c_int32, C.c_int64, C.c_void_p, C.c_size_t
        lib.gllm_op_tree_attention.restype = i32
        lib.gllm_op_tree_attention.argtypes = [vp, i64, vp, vp, i64, vp, i32, vp, vp, vp, i32, i32, i32, i32, i32, i32, C.c_float, vp, i64,
                                               vp, sz, vp]
        lib.gllm_op_tree_attention_workspace_bytes.restype = sz
        lib.gllm_op_tree_attention_workspace_bytes.argtypes = [i32, i32, i32, i32]
        lib.gllm_op_tree_commit.restype = i32
        lib.gllm_op_tree_commit.argtypes = [vp, vp, vp, vp, vp, vp, i32, i32, i32, vp, vp, i32, i64, i32, i32, vp, vp, vp, vp]
        lib.gllm_op_beam_select.restype = i32
        lib.gllm_op_beam_select.argtypes = [vp, i64, vp, i32, i32, i32, i32, vp, vp, vp, vp, sz, vp]
        lib.gllm_op_beam_select_workspace_bytes.restype = sz
        lib.gllm_op_beam_select_workspace_bytes.argtypes = [i32, i32, i32, i32]
        lib.gllm_op_copy_pages.restype = i32
        lib.gllm_op_copy_pages.argtypes = [vp, vp, i32, i64, i32, i32, vp, vp, i32, vp]
        _ready = lib
    return _ready


def _refuse(what: str):
    raise GllmError(_INVALID, what)


_BF16, _F32, _I32, _U8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8


def _check(call: str, tensors, rows_only=()) -> int:
    """tensors: pairs of a tensor and its type, all on the current GPU and contiguous (those of rows_only: inside a row).  Returns the
    GPU's index."""
    dev = tensors[0][0].get_device()
    if dev < 0 or dev != torch._C._cuda_getDevice():           # (what torch.cuda.current_device() asks, behind a look at the environment)
        _refuse(f"{call}: tensors on the current GPU are wanted, got one on {tensors[0][0].device}")
    for t, dtype in tensors:
        if t.get_device() != dev or t.dtype is not dtype:
            _refuse(f"{call}: a tensor of {dtype} on cuda:{dev} is wanted, got {t.dtype} on {t.device}")
        if not t.is_contiguous():
            for r in rows_only:
                if r is t and t.dim() == 2 and t.stride(1) == 1:
                    break
            else:
                _refuse(f"{call}: a tensor of shape {tuple(t.shape)} and strides {t.stride()} is not contiguous")
    return dev


def _stream(stream, dev: int) -> int:
    return torch._C._cuda_getCurrentRawStream(dev) if stream is None else _stream_ptr(stream)


def _own_workspace(call: str, size: int, like, stream):
    """A workspace from torch's allocator, which may give it to somebody else on the call's stream only."""
    if stream is None:
        return torch.empty(size, dtype=torch.uint8, device=like.device)
    if isinstance(stream, int):
        _refuse(f"{call}: a stream given by its handle needs a workspace of the caller's")
    with torch.cuda.stream(stream):
        return torch.empty(size, dtype=torch.uint8, device=like.device)


def _row_stride(t) -> int:
    """The row stride of a 2-d tensor (torch gives a tensor of one row any)."""
    return t.stride(0) if t.shape[0] > 1 else max(t.stride(0), t.shape[1])


def _pool_shape(call: str, k_pool, v_pool, dims: int):
    """(KV heads, head size) of pools [.., n_kv, d/8, 16, 8] and [.., n_kv, d, 16] with `dims` dimensions in front."""
    k, v = k_pool.shape, v_pool.shape
    if len(k) != dims + 4 or len(v) != dims + 3 or k[:dims + 1] != v[:dims + 1] or k[-1] != 8 or k[-2] != PAGE or v[-1] != PAGE or v[-2] != 8 * k[-3] or v[-2] == 0:
        _refuse(f"{call}: pools of shapes {tuple(k)} and {tuple(v)}")
    return k[dims], v[-2]


def gllm_op_tree_attention_workspace_bytes(n_q_heads: int, n_kv_heads: int, head_dim: int, max_nodes: int) -> int:
    return int(_lib().gllm_op_tree_attention_workspace_bytes(n_q_heads, n_kv_heads, head_dim, max_nodes))


def gllm_op_tree_attention(q, k_pool, v_pool, block_tables, cached_len, row_start, parents, out, max_nodes: int, scale=None,
                           workspace=None, stream=None) -> None:
    """q, out: bf16 [R, n_q*d]; k_pool: bf16 [pages, n_kv, d/8, 16, 8], v_pool: bf16 [pages, n_kv, d, 16], one layer; block_tables:
    int32 [S, entries]; cached_len: int32 [S]; row_start: int32 [S+1]; parents: int32 [R].  scale: 1/sqrt(d) if not given;
    workspace: uint8, taken from torch's allocator if not given."""
    call = "gllm_op_tree_attention"
    n_kv, d = _pool_shape(call, k_pool, v_pool, 1)
    dev = _check(call, ((q, _BF16), (out, _BF16), (k_pool, _BF16), (v_pool, _BF16), (block_tables, _I32), (cached_len, _I32), (row_start, _I32),
                        (parents, _I32)), rows_only=(q, out))
    rows, seqs = parents.numel(), cached_len.numel()
    if q.dim() != 2 or q.shape[0] != rows or cached_len.dim() < 1 or q.shape[1] % d != 0 or out.shape != q.shape or block_tables.dim() != 2 or block_tables.shape[0] != seqs or row_start.numel() != seqs + 1:
        _refuse(f"{call}: shapes q {tuple(q.shape)}, out {tuple(out.shape)}, block_tables {tuple(block_tables.shape)}, cached_len {tuple(cached_len.shape)}, "
                f"row_start {tuple(row_start.shape)}, parents {tuple(parents.shape)}")
    n_q = q.shape[1] // d
    lib = _lib()
    if workspace is None:
        workspace = _own_workspace(call, int(lib.gllm_op_tree_attention_workspace_bytes(n_q, n_kv, d, max_nodes)), q, stream)
    _check(call, ((workspace, _U8),))
    st = lib.gllm_op_tree_attention(q.data_ptr(), _row_stride(q), k_pool.data_ptr(), v_pool.data_ptr(), k_pool.shape[0], block_tables.data_ptr(),
                                    block_tables.shape[1], cached_len.data_ptr(), row_start.data_ptr(), parents.data_ptr(), seqs, rows,
                                    max_nodes, n_q, n_kv, d, 1.0 / math.sqrt(d) if scale is None else scale, out.data_ptr(), _row_stride(out),
                                    workspace.data_ptr(), workspace.numel(), _stream(stream, dev))
    if st != GLLM_OK:
        raise GllmError(st, call)


def gllm_op_tree_commit(tokens, parents, sampled, row_start, cached_len, block_tables, k_pool, v_pool, path, count, next_token,
                        stream=None) -> None:
    """tokens, parents, sampled, path: int32 [R]; row_start: int32 [S+1]; cached_len, count, next_token: int32 [S]; block_tables: int32
    [S, entries]; k_pool: bf16 [layers, pages, n_kv, d/8, 16, 8], v_pool: bf16 [layers, pages, n_kv, d, 16], or both None (no moves)."""
    call = "gllm_op_tree_commit"
    dev = _check(call, ((tokens, _I32), (parents, _I32), (sampled, _I32), (path, _I32), (row_start, _I32), (cached_len, _I32), (block_tables, _I32),
                        (count, _I32), (next_token, _I32)))
    rows, seqs = tokens.numel(), cached_len.numel()
    if parents.numel() != rows or sampled.numel() != rows or path.numel() != rows or row_start.numel() != seqs + 1 or block_tables.dim() != 2 or \
            block_tables.shape[0] != seqs or count.numel() != seqs or next_token.numel() != seqs or (k_pool is None) != (v_pool is None):
        _refuse(f"{call}: arrays of {rows} rows and {seqs} sequences do not fit each other")
    layers = pages = n_kv = d = 0
    if k_pool is not None:
        n_kv, d = _pool_shape(call, k_pool, v_pool, 2)
        _check(call, ((k_pool, _BF16), (v_pool, _BF16)))
        layers, pages = k_pool.shape[:2]
    st = _lib().gllm_op_tree_commit(tokens.data_ptr(), parents.data_ptr(), sampled.data_ptr(), row_start.data_ptr(), cached_len.data_ptr(),
                                    block_tables.data_ptr(), block_tables.shape[1], seqs, rows, None if k_pool is None else k_pool.data_ptr(),
                                    None if v_pool is None else v_pool.data_ptr(), layers, pages, n_kv, d, path.data_ptr(), count.data_ptr(),
                                    next_token.data_ptr(), _stream(stream, dev))
    if st != GLLM_OK:
        raise GllmError(st, call)


def gllm_op_beam_select_workspace_bytes(num_seqs: int, beams: int, vocab: int, keep: int) -> int:
    return int(_lib().gllm_op_beam_select_workspace_bytes(num_seqs, beams, vocab, keep))


def gllm_op_beam_select(logits, vocab: int, scores, out_scores, out_beams, out_tokens, workspace=None, stream=None) -> None:
    """logits: fp32 [S*W, >= vocab] (row stride taken from the tensor); scores: fp32 [S, W]; out_scores: fp32, out_beams, out_tokens:
    int32, [S, keep]; workspace: uint8, taken from torch's allocator if not given."""
    call = "gllm_op_beam_select"
    dev = _check(call, ((logits, _F32), (scores, _F32), (out_scores, _F32), (out_beams, _I32), (out_tokens, _I32)), rows_only=(logits,))
    if logits.dim() != 2 or scores.dim() != 2 or out_scores.dim() != 2 or logits.shape[0] != scores.numel() or logits.shape[1] < vocab or out_scores.shape[0] != scores.shape[0] or \
            out_beams.shape != out_scores.shape or out_tokens.shape != out_scores.shape:
        _refuse(f"{call}: shapes logits {tuple(logits.shape)}, scores {tuple(scores.shape)}, outputs {tuple(out_scores.shape)}, "
                f"{tuple(out_beams.shape)}, {tuple(out_tokens.shape)}, vocabulary {vocab}")
    lib = _lib()
    seqs, beams, keep = scores.shape[0], scores.shape[1], out_scores.shape[1]
    if workspace is None:
        workspace = _own_workspace(call, int(lib.gllm_op_beam_select_workspace_bytes(seqs, beams, vocab, keep)), logits, stream)
    _check(call, ((workspace, _U8),))
    st = lib.gllm_op_beam_select(logits.data_ptr(), _row_stride(logits), scores.data_ptr(), seqs, beams, vocab, keep, out_scores.data_ptr(),
                                 out_beams.data_ptr(), out_tokens.data_ptr(), workspace.data_ptr(), workspace.numel(), _stream(stream, dev))
    if st != GLLM_OK:
        raise GllmError(st, call)


def _page_ids(call: str, ids):
    """(address, number, owner of the memory) of int32 page ids; what is no whole number of 32 bits is refused, not cut to one."""
    if type(ids) is list:
        try:
            a = array("i", ids)
            return *a.buffer_info(), a
        except (TypeError, OverflowError):
            pass
    try:
        given = np.asarray(ids)
    except (TypeError, ValueError):
        _refuse(f"{call}: page ids are whole numbers on the host, got {type(ids).__name__}")
    if given.dtype.kind in "iu":
        a = np.ascontiguousarray(given, dtype=np.int32)
        if a is not given and not (a == given).all():
            raise GllmError(_BLOCK_RANGE, f"{call}: page ids outside the pool")
    else:
        if given.size > 0 and given.dtype.kind != "f" and not all(isinstance(x, int) for x in given.flat):
            _refuse(f"{call}: page ids are whole numbers, got an array of {given.dtype}")
        if given.dtype.kind == "f" and not (given == np.floor(given)).all():
            _refuse(f"{call}: page ids are whole numbers")
        if given.size > 0 and not -2 ** 31 <= given.min() <= given.max() < 2 ** 31:
            raise GllmError(_BLOCK_RANGE, f"{call}: page ids outside the pool")
        a = np.ascontiguousarray(given, dtype=np.int32)
    if given.ndim != 1:
        _refuse(f"{call}: page ids of shape {given.shape}")
    return a.ctypes.data, a.shape[0], a


def gllm_op_copy_pages(k_pool, v_pool, src, dst, stream=None) -> None:
    """k_pool: bf16 [layers, pages, n_kv, d/8, 16, 8], v_pool: bf16 [layers, pages, n_kv, d, 16]; src, dst: page ids on the host."""
    call = "gllm_op_copy_pages"
    n_kv, d = _pool_shape(call, k_pool, v_pool, 2)
    (s, n, _s), (t, n_dst, _t) = _page_ids(call, src), _page_ids(call, dst)
    dev = _check(call, ((k_pool, _BF16), (v_pool, _BF16)))
    if n != n_dst:
        _refuse(f"{call}: {n} sources, {n_dst} destinations")
    st = _lib().gllm_op_copy_pages(k_pool.data_ptr(), v_pool.data_ptr(), k_pool.shape[0], k_pool.shape[1], n_kv, d, s, t, n, _stream(stream, dev))
    if st != GLLM_OK:
        raise GllmError(st, call)
