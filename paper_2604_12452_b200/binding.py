"""Thin ctypes binding of the LCA C ABI (include/lca.h).

The functions named ``lca_*`` take the same arguments as the C entry points; tensors may be
passed as torch tensors (their device pointer is taken), raw integer addresses, or None.  They
return the integer status.  The helpers below them (``condense``, ``prefill_attention``,
``decode_attention``) only allocate outputs / workspace with torch and check the status; every
step of the method runs inside the CUDA library.  There is no CPU fallback: importing this
module without the built library raises.
"""
from __future__ import annotations

import ctypes as C
import math
import os
from typing import Optional

import torch

from . import build as _build

LCA_OK = 0
LCA_VARIANT_MLA, LCA_VARIANT_GQA = 0, 1
LCA_WS_CONDENSE, LCA_WS_PREFILL, LCA_WS_DECODE, LCA_WS_UPDATE = 0, 1, 2, 3
LCA_WS_CONDENSE_VARLEN, LCA_WS_PREFILL_VARLEN = 4, 5
LCA_STATIC_SCRATCH_BYTES = 1 << 20
LCA_ERR_STATIC_SCRATCH_EXCEEDED = -7
LCA_ERR_DEVICE_TIMEOUT = -6
ATTN_AUTO, ATTN_SCALAR, ATTN_TENSOR = 0, 1, 2
LCA_DTYPE_BF16, LCA_DTYPE_FP32 = 0, 1
ROPE_PLAIN, ROPE_LINEAR, ROPE_BASE, ROPE_RAMP = 0, 1, 2, 3
REDUCE_DEFAULT, REDUCE_MAXPOOL, REDUCE_MEANPOOL, REDUCE_WEIGHTED, REDUCE_MAXSEL = 0, 1, 2, 3, 4


class LcaParams(C.Structure):
    """Mirror of ``lca_params`` (Alg. 1 REQUIRE line + head layout)."""
    _fields_ = [("variant", C.c_int32), ("batch", C.c_int32), ("seq_len", C.c_int32),
                ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("d_sem", C.c_int32),
                ("d_pos", C.c_int32), ("group_size", C.c_int32), ("window", C.c_int32),
                ("n_summary_q", C.c_int32), ("softmax_scale", C.c_float),
                ("rep_logit_bias", C.c_float), ("sem_reducer", C.c_int32), ("pos_reducer", C.c_int32)]


class LcaPaged8(C.Structure):
    """Mirror of ``lca_paged8``: device pointers of a paged 8-bit cache.  Build it with ``paged8_cache``, which also keeps
    the tensors alive."""
    _fields_ = [("pages_sem", C.c_void_p), ("pages_pos", C.c_void_p), ("scale_sem", C.c_void_p), ("scale_pos", C.c_void_p),
                ("block_table", C.c_void_p), ("n_pages", C.c_int32), ("page_size", C.c_int32), ("table_width", C.c_int32)]
    tensors: tuple = ()
    device: Optional[int] = None               # CUDA device of the tensors (-1: not on one)
    batch: Optional[int] = None                # rows of block_table
    layout: Optional[tuple] = None             # (n_kv_heads, d_sem, d_pos) of the pages


class LcaPaged4(C.Structure):
    """Mirror of ``lca_paged4``: device pointers of a paged 4-bit cache.  Build it with ``paged4_cache``, which also keeps
    the tensors alive."""
    _fields_ = [("pages_sem", C.c_void_p), ("pages_pos", C.c_void_p), ("shift_sem", C.c_void_p), ("shift_pos", C.c_void_p),
                ("exp_sem", C.c_void_p), ("exp_pos", C.c_void_p), ("block_table", C.c_void_p), ("n_pages", C.c_int32),
                ("page_size", C.c_int32), ("table_width", C.c_int32)]
    tensors: tuple = ()
    device: Optional[int] = None
    batch: Optional[int] = None
    layout: Optional[tuple] = None
    pages: Optional[LcaPaged8] = None          # the same tables for lca_page_update, which manages the pages of either cache


class LcaRopeArgs(C.Structure):
    """Mirror of ``lca_rope_args``."""
    _fields_ = [("dtype", C.c_int32), ("interleaved", C.c_int32), ("inverse", C.c_int32), ("n_q_heads", C.c_int32),
                ("n_k_heads", C.c_int32), ("head_dim", C.c_int32), ("rot_dim", C.c_int32), ("factor", C.c_float),
                ("n_tokens", C.c_int64), ("positions", C.c_void_p), ("freqs", C.c_void_p),
                ("q", C.c_void_p), ("q_token_stride", C.c_int64), ("q_head_stride", C.c_int64),
                ("q_out", C.c_void_p), ("q_out_token_stride", C.c_int64), ("q_out_head_stride", C.c_int64),
                ("k", C.c_void_p), ("k_token_stride", C.c_int64), ("k_head_stride", C.c_int64),
                ("k_out", C.c_void_p), ("k_out_token_stride", C.c_int64), ("k_out_head_stride", C.c_int64)]


class LcaVerifyArgs(C.Structure):
    """Mirror of ``lca_verify_args``."""
    _fields_ = [("dtype", C.c_int32), ("batch", C.c_int32), ("n_drafts", C.c_int32), ("vocab", C.c_int32),
                ("target_probs", C.c_void_p), ("draft_probs", C.c_void_p), ("draft_tokens", C.c_void_p), ("n_draft", C.c_void_p),
                ("u_accept", C.c_void_p), ("u_sample", C.c_void_p), ("n_tok", C.c_void_p), ("accepted", C.c_void_p),
                ("tokens_out", C.c_void_p), ("n_tok_out", C.c_void_p)]


class LcaError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {lca_status_string(status)} ({status})")


def _load() -> C.CDLL:
    path = _build.LIB
    if not os.path.exists(path):
        raise ImportError(f"{path} is missing: build it with paper_2604_12452_b200.build.build() "
                          "(python __graft_entry__.py); there is no fallback path")
    lib = C.CDLL(path)
    vp, i32, i64, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
    P = C.POINTER(LcaParams)
    lib.lca_version.restype = C.c_int
    lib.lca_status_string.restype = C.c_char_p
    lib.lca_status_string.argtypes = [C.c_int]
    lib.lca_launch_count.restype = i64
    lib.lca_set_attention_impl.restype = C.c_int
    lib.lca_set_attention_impl.argtypes = [C.c_int]
    lib.lca_partition.restype = C.c_int
    lib.lca_partition.argtypes = [P, C.POINTER(i32), C.POINTER(i32)]
    lib.lca_workspace_bytes.restype = sz
    lib.lca_workspace_bytes.argtypes = [P, i32]
    lib.lca_condense.restype = C.c_int
    lib.lca_condense.argtypes = [P, vp, vp, i64, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.lca_condense_static_scratch.restype = C.c_int
    lib.lca_condense_static_scratch.argtypes = [P, vp, vp, i64, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.lca_prefill_attention.restype = C.c_int
    lib.lca_prefill_attention.argtypes = [P, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.lca_decode_attention.restype = C.c_int
    lib.lca_decode_attention.argtypes = [P, vp, vp, vp, vp, vp, i32, i32, vp, vp, vp, sz, vp]
    lib.lca_decode_update.restype = C.c_int
    lib.lca_decode_update.argtypes = [P, vp, vp, i64, vp, vp, vp, i32, vp, vp, vp, vp, sz, vp]
    lib.lca_ring_from_packed.restype = C.c_int
    lib.lca_ring_from_packed.argtypes = [P, vp, vp, vp, vp, i32, vp, vp, i32, vp, vp]
    lib.lca_decode_attention_ring.restype = C.c_int
    lib.lca_decode_attention_ring.argtypes = [P, vp, vp, vp, vp, vp, vp, i32, vp, vp, vp, sz, vp]
    lib.lca_decode_update_ring.restype = C.c_int
    lib.lca_decode_update_ring.argtypes = [P, vp, vp, i64, vp, vp, vp, i32, vp, vp, vp, vp, sz, vp]
    lib.lca_decode_step_update_ring.restype = C.c_int
    lib.lca_decode_step_update_ring.argtypes = [P, vp, vp, vp, vp, vp, vp, i32, vp, vp, vp, vp, sz, vp]
    pi32, pi64 = C.POINTER(i32), C.POINTER(i64)
    lib.lca_varlen_layout.restype = C.c_int
    lib.lca_varlen_layout.argtypes = [P, pi32, pi64, pi64, pi64]
    lib.lca_condense_varlen.restype = C.c_int
    lib.lca_condense_varlen.argtypes = [P, pi32, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.lca_prefill_attention_varlen.restype = C.c_int
    lib.lca_prefill_attention_varlen.argtypes = [P, pi32, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    PC = C.POINTER(LcaPaged8)
    lib.lca_page_update.restype = C.c_int
    lib.lca_page_update.argtypes = [P, PC, vp, vp, vp, vp, vp, vp, vp, i32, i32, vp, vp, vp]
    lib.lca_paged8_write.restype = C.c_int
    lib.lca_paged8_write.argtypes = [P, PC, vp, vp, vp, i64, vp]
    lib.lca_paged8_workspace_bytes.restype = sz
    lib.lca_paged8_workspace_bytes.argtypes = [P, PC, i32]
    lib.lca_decode_attention_paged8.restype = C.c_int
    lib.lca_decode_attention_paged8.argtypes = [P, PC, vp, vp, i32, vp, vp, vp, vp, vp, sz, vp]
    lib.lca_decode_update_paged8.restype = C.c_int
    lib.lca_decode_update_paged8.argtypes = [P, PC, vp, vp, i64, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    P4 = C.POINTER(LcaPaged4)
    lib.lca_paged4_write.restype = C.c_int
    lib.lca_paged4_write.argtypes = [P, P4, vp, vp, vp, i64, vp]
    lib.lca_paged4_read.restype = C.c_int
    lib.lca_paged4_read.argtypes = [P, P4, vp, vp, vp, i64, vp]
    lib.lca_paged4_workspace_bytes.restype = sz
    lib.lca_paged4_workspace_bytes.argtypes = [P, P4, i32]
    lib.lca_decode_attention_paged4.restype = C.c_int
    lib.lca_decode_attention_paged4.argtypes = [P, P4, vp, vp, i32, vp, vp, vp, vp, vp, sz, vp]
    lib.lca_decode_update_paged4.restype = C.c_int
    lib.lca_decode_update_paged4.argtypes = [P, P4, vp, vp, i64, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.lca_rope.restype = C.c_int
    lib.lca_rope.argtypes = [C.POINTER(LcaRopeArgs), vp]
    lib.lca_rope_frequencies.restype = C.c_int
    lib.lca_rope_frequencies.argtypes = [i32, i32] + [C.c_double] * 5 + [C.POINTER(C.c_double), C.POINTER(C.c_float)]
    lib.lca_verify_drafts.restype = C.c_int
    lib.lca_verify_drafts.argtypes = [C.POINTER(LcaVerifyArgs), vp]
    lib.lca_latent_to_value.restype = C.c_int
    lib.lca_latent_to_value.argtypes = [vp, vp, vp, i64, i32, i32, i32, vp]
    lib.lca_selftest_bounded_wait.restype = C.c_int
    lib.lca_selftest_bounded_wait.argtypes = [i64, vp]
    lib.lca_last_device_status.restype = C.c_int
    lib.lca_last_device_status.argtypes = [vp]
    return lib


_lib = _load()


def _ptr(x):
    if x is None:
        return None
    if isinstance(x, torch.Tensor):
        if not x.is_contiguous():
            raise ValueError("the LCA entry points take dense row-major tensors: call .contiguous() first")
        return x.data_ptr()
    return int(x)


def _nbytes(x) -> int:
    return 0 if x is None else x.numel() * x.element_size()


_has_cuda: Optional[bool] = None


def _stream(stream):
    if stream is None:
        global _has_cuda
        if _has_cuda is None:                  # asked once: the answer costs more than a small call's launch
            _has_cuda = torch.cuda.is_available()
        if not _has_cuda:                      # host-side validation calls on a GPU-less machine
            return 0
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    if isinstance(stream, torch.cuda.Stream):
        return stream.cuda_stream
    return int(stream)


# ------------------------------------------------------------------ raw entry points (same names)
def lca_version() -> int:
    return int(_lib.lca_version())


def lca_status_string(status: int) -> str:
    return _lib.lca_status_string(int(status)).decode()


def lca_launch_count() -> int:
    return int(_lib.lca_launch_count())


def lca_set_attention_impl(impl: int) -> int:
    return int(_lib.lca_set_attention_impl(int(impl)))


def lca_partition(params: LcaParams):
    m, k = C.c_int32(), C.c_int32()
    st = _lib.lca_partition(C.byref(params), C.byref(m), C.byref(k))
    if st != LCA_OK:
        raise LcaError(st, "lca_partition")
    return int(m.value), int(k.value)


def lca_workspace_bytes(params: LcaParams, which: int) -> int:
    return int(_lib.lca_workspace_bytes(C.byref(params), int(which)))


def lca_condense(params, q_tail_sem, q_tail_pos, q_tail_batch_stride, qbar_opt, kv_sem, kv_pos,
                 cache_sem, cache_pos, anchor_idx, scores_opt, ws, ws_bytes=None, stream=None) -> int:
    wsb = _nbytes(ws) if ws_bytes is None else int(ws_bytes)
    return int(_lib.lca_condense(C.byref(params), _ptr(q_tail_sem), _ptr(q_tail_pos),
                                 int(q_tail_batch_stride), _ptr(qbar_opt), _ptr(kv_sem), _ptr(kv_pos),
                                 _ptr(cache_sem), _ptr(cache_pos), _ptr(anchor_idx), _ptr(scores_opt),
                                 _ptr(ws), wsb, _stream(stream)))


def lca_condense_static_scratch(params, q_tail_sem, q_tail_pos, q_tail_batch_stride, qbar_opt, kv_sem,
                                kv_pos, cache_sem, cache_pos, anchor_idx, scores_opt, stream=None) -> int:
    """lca_condense without a workspace argument: the scratch is a fixed array inside the library
    (for callers that must not allocate device memory).  Same outputs, bit for bit."""
    return int(_lib.lca_condense_static_scratch(C.byref(params), _ptr(q_tail_sem), _ptr(q_tail_pos),
                                                int(q_tail_batch_stride), _ptr(qbar_opt), _ptr(kv_sem),
                                                _ptr(kv_pos), _ptr(cache_sem), _ptr(cache_pos),
                                                _ptr(anchor_idx), _ptr(scores_opt), _stream(stream)))


def lca_prefill_attention(params, q_sem, q_pos, kv_sem, kv_pos, cache_sem, cache_pos, out, lse_opt,
                          ws, ws_bytes=None, stream=None) -> int:
    wsb = _nbytes(ws) if ws_bytes is None else int(ws_bytes)
    return int(_lib.lca_prefill_attention(C.byref(params), _ptr(q_sem), _ptr(q_pos), _ptr(kv_sem),
                                          _ptr(kv_pos), _ptr(cache_sem), _ptr(cache_pos), _ptr(out),
                                          _ptr(lse_opt), _ptr(ws), wsb, _stream(stream)))


def lca_decode_attention(params, q_sem, q_pos, cache_sem, cache_pos, cache_rows, cache_row_capacity,
                         n_rep, out, lse_opt, ws, ws_bytes=None, stream=None) -> int:
    wsb = _nbytes(ws) if ws_bytes is None else int(ws_bytes)
    return int(_lib.lca_decode_attention(C.byref(params), _ptr(q_sem), _ptr(q_pos), _ptr(cache_sem),
                                         _ptr(cache_pos), _ptr(cache_rows), int(cache_row_capacity),
                                         int(n_rep), _ptr(out), _ptr(lse_opt), _ptr(ws), wsb,
                                         _stream(stream)))


def lca_decode_update(params, q_tail_sem, q_tail_pos, q_tail_batch_stride, qbar_opt, cache_sem, cache_pos,
                      cache_row_capacity, n_rep, cache_rows, anchor_out, ws, ws_bytes=None, stream=None) -> int:
    wsb = _nbytes(ws) if ws_bytes is None else int(ws_bytes)
    return int(_lib.lca_decode_update(C.byref(params), _ptr(q_tail_sem), _ptr(q_tail_pos), int(q_tail_batch_stride),
                                      _ptr(qbar_opt), _ptr(cache_sem), _ptr(cache_pos), int(cache_row_capacity),
                                      _ptr(n_rep), _ptr(cache_rows), _ptr(anchor_out), _ptr(ws), wsb, _stream(stream)))


def lca_ring_from_packed(params, packed_sem, packed_pos, packed_rows, n_rep, packed_row_capacity, ring_sem, ring_pos,
                         ring_row_capacity, n_tok_out, stream=None) -> int:
    return int(_lib.lca_ring_from_packed(C.byref(params), _ptr(packed_sem), _ptr(packed_pos), _ptr(packed_rows), _ptr(n_rep),
                                         int(packed_row_capacity), _ptr(ring_sem), _ptr(ring_pos), int(ring_row_capacity),
                                         _ptr(n_tok_out), _stream(stream)))


def lca_decode_attention_ring(params, q_sem, q_pos, ring_sem, ring_pos, n_rep, n_tok, ring_row_capacity, out, lse_opt,
                              ws, ws_bytes=None, stream=None) -> int:
    wsb = _nbytes(ws) if ws_bytes is None else int(ws_bytes)
    return int(_lib.lca_decode_attention_ring(C.byref(params), _ptr(q_sem), _ptr(q_pos), _ptr(ring_sem), _ptr(ring_pos),
                                              _ptr(n_rep), _ptr(n_tok), int(ring_row_capacity), _ptr(out), _ptr(lse_opt),
                                              _ptr(ws), wsb, _stream(stream)))


def lca_decode_update_ring(params, q_tail_sem, q_tail_pos, q_tail_batch_stride, qbar_opt, ring_sem, ring_pos,
                           ring_row_capacity, n_rep, n_tok, anchor_out, ws, ws_bytes=None, stream=None) -> int:
    wsb = _nbytes(ws) if ws_bytes is None else int(ws_bytes)
    return int(_lib.lca_decode_update_ring(C.byref(params), _ptr(q_tail_sem), _ptr(q_tail_pos), int(q_tail_batch_stride),
                                           _ptr(qbar_opt), _ptr(ring_sem), _ptr(ring_pos), int(ring_row_capacity),
                                           _ptr(n_rep), _ptr(n_tok), _ptr(anchor_out), _ptr(ws), wsb, _stream(stream)))


def lca_decode_step_update_ring(params, q_sem, q_pos, qsum, qcount, ring_sem, ring_pos, ring_row_capacity, n_rep, n_tok,
                                anchor_out, ws, ws_bytes=None, stream=None) -> int:
    wsb = _nbytes(ws) if ws_bytes is None else int(ws_bytes)
    return int(_lib.lca_decode_step_update_ring(C.byref(params), _ptr(q_sem), _ptr(q_pos), _ptr(qsum), _ptr(qcount),
                                                _ptr(ring_sem), _ptr(ring_pos), int(ring_row_capacity), _ptr(n_rep),
                                                _ptr(n_tok), _ptr(anchor_out), _ptr(ws), wsb, _stream(stream)))


def _lens(seq_lens):
    return (C.c_int32 * len(seq_lens))(*[int(x) for x in seq_lens])


def lca_varlen_layout(params, seq_lens):
    """(token_offsets, cache_row_offsets, group_offsets): lists of batch + 1 prefix sums."""
    n = params.batch + 1
    tok, cache, grp = (C.c_int64 * n)(), (C.c_int64 * n)(), (C.c_int64 * n)()
    st = _lib.lca_varlen_layout(C.byref(params), _lens(seq_lens), tok, cache, grp)
    if st != LCA_OK:
        raise LcaError(st, "lca_varlen_layout")
    return list(tok), list(cache), list(grp)


def lca_condense_varlen(params, seq_lens, q_sem, q_pos, qbar_opt, kv_sem, kv_pos, cache_sem, cache_pos, anchor_idx,
                        ws, ws_bytes=None, stream=None) -> int:
    wsb = _nbytes(ws) if ws_bytes is None else int(ws_bytes)
    return int(_lib.lca_condense_varlen(C.byref(params), _lens(seq_lens), _ptr(q_sem), _ptr(q_pos), _ptr(qbar_opt),
                                        _ptr(kv_sem), _ptr(kv_pos), _ptr(cache_sem), _ptr(cache_pos), _ptr(anchor_idx),
                                        _ptr(ws), wsb, _stream(stream)))


def lca_prefill_attention_varlen(params, seq_lens, q_sem, q_pos, kv_sem, kv_pos, cache_sem, cache_pos, out, lse_opt,
                                 ws, ws_bytes=None, stream=None) -> int:
    wsb = _nbytes(ws) if ws_bytes is None else int(ws_bytes)
    return int(_lib.lca_prefill_attention_varlen(C.byref(params), _lens(seq_lens), _ptr(q_sem), _ptr(q_pos), _ptr(kv_sem),
                                                 _ptr(kv_pos), _ptr(cache_sem), _ptr(cache_pos), _ptr(out), _ptr(lse_opt),
                                                 _ptr(ws), wsb, _stream(stream)))


def lca_page_update(params, cache, n_rep, n_tok, held_rep, held_tok, free_pages, n_free, slot_map, n_rows, rows_per_seq,
                    row_offsets, status, stream=None) -> int:
    return int(_lib.lca_page_update(C.byref(params), C.byref(cache), _ptr(n_rep), _ptr(n_tok), _ptr(held_rep), _ptr(held_tok),
                                    _ptr(free_pages), _ptr(n_free), _ptr(slot_map), int(n_rows), int(rows_per_seq),
                                    _ptr(row_offsets), _ptr(status), _stream(stream)))


def lca_paged8_write(params, cache, rows_sem, rows_pos, slot_map, n_rows, stream=None) -> int:
    return int(_lib.lca_paged8_write(C.byref(params), C.byref(cache), _ptr(rows_sem), _ptr(rows_pos), _ptr(slot_map), int(n_rows),
                                     _stream(stream)))


def lca_paged8_workspace_bytes(params, cache, q_len: int) -> int:
    return int(_lib.lca_paged8_workspace_bytes(C.byref(params), C.byref(cache), int(q_len)))


def lca_decode_attention_paged8(params, cache, q_sem, q_pos, q_len, n_rep, n_tok, out, lse_opt, ws, ws_bytes=None, stream=None) -> int:
    wsb = _nbytes(ws) if ws_bytes is None else int(ws_bytes)
    return int(_lib.lca_decode_attention_paged8(C.byref(params), C.byref(cache), _ptr(q_sem), _ptr(q_pos), int(q_len), _ptr(n_rep),
                                                _ptr(n_tok), _ptr(out), _ptr(lse_opt), _ptr(ws), wsb, _stream(stream)))


def lca_decode_update_paged8(params, cache, q_tail_sem, q_tail_pos, q_tail_batch_stride, qbar_opt, n_rep, n_tok, n_rep_new, rep_sem,
                             rep_pos, anchor_out, ws, ws_bytes=None, stream=None) -> int:
    wsb = _nbytes(ws) if ws_bytes is None else int(ws_bytes)
    return int(_lib.lca_decode_update_paged8(C.byref(params), C.byref(cache), _ptr(q_tail_sem), _ptr(q_tail_pos),
                                             int(q_tail_batch_stride), _ptr(qbar_opt), _ptr(n_rep), _ptr(n_tok), _ptr(n_rep_new),
                                             _ptr(rep_sem), _ptr(rep_pos), _ptr(anchor_out), _ptr(ws), wsb, _stream(stream)))


def lca_paged4_write(params, cache, rows_sem, rows_pos, slot_map, n_rows, stream=None) -> int:
    return int(_lib.lca_paged4_write(C.byref(params), C.byref(cache), _ptr(rows_sem), _ptr(rows_pos), _ptr(slot_map), int(n_rows),
                                     _stream(stream)))


def lca_paged4_read(params, cache, rows_sem, rows_pos, slot_map, n_rows, stream=None) -> int:
    return int(_lib.lca_paged4_read(C.byref(params), C.byref(cache), _ptr(rows_sem), _ptr(rows_pos), _ptr(slot_map), int(n_rows),
                                    _stream(stream)))


def lca_paged4_workspace_bytes(params, cache, q_len: int) -> int:
    return int(_lib.lca_paged4_workspace_bytes(C.byref(params), C.byref(cache), int(q_len)))


def lca_decode_attention_paged4(params, cache, q_sem, q_pos, q_len, n_rep, n_tok, out, lse_opt, ws, ws_bytes=None, stream=None) -> int:
    wsb = _nbytes(ws) if ws_bytes is None else int(ws_bytes)
    return int(_lib.lca_decode_attention_paged4(C.byref(params), C.byref(cache), _ptr(q_sem), _ptr(q_pos), int(q_len), _ptr(n_rep),
                                                _ptr(n_tok), _ptr(out), _ptr(lse_opt), _ptr(ws), wsb, _stream(stream)))


def lca_decode_update_paged4(params, cache, q_tail_sem, q_tail_pos, q_tail_batch_stride, qbar_opt, n_rep, n_tok, n_rep_new, rep_sem,
                             rep_pos, anchor_out, ws, ws_bytes=None, stream=None) -> int:
    wsb = _nbytes(ws) if ws_bytes is None else int(ws_bytes)
    return int(_lib.lca_decode_update_paged4(C.byref(params), C.byref(cache), _ptr(q_tail_sem), _ptr(q_tail_pos),
                                             int(q_tail_batch_stride), _ptr(qbar_opt), _ptr(n_rep), _ptr(n_tok), _ptr(n_rep_new),
                                             _ptr(rep_sem), _ptr(rep_pos), _ptr(anchor_out), _ptr(ws), wsb, _stream(stream)))


def lca_rope(args: LcaRopeArgs, stream=None) -> int:
    return int(_lib.lca_rope(C.byref(args), _stream(stream)))


def lca_rope_frequencies(kind, rot_dim, base, scale, trained_len, fast, slow, freqs, factor) -> int:
    """``freqs``: a ctypes array of rot_dim / 2 doubles, ``factor`` a c_float, both filled in."""
    return int(_lib.lca_rope_frequencies(int(kind), int(rot_dim), base, scale, trained_len, fast, slow, freqs,
                                         None if factor is None else C.byref(factor)))


def lca_verify_drafts(args: LcaVerifyArgs, stream=None) -> int:
    return int(_lib.lca_verify_drafts(C.byref(args), _stream(stream)))


def lca_latent_to_value(attn_latent, w_uv, out_v, n_tokens, n_heads, d_latent, d_v, stream=None) -> int:
    return int(_lib.lca_latent_to_value(_ptr(attn_latent), _ptr(w_uv), _ptr(out_v), int(n_tokens), int(n_heads),
                                        int(d_latent), int(d_v), _stream(stream)))


def lca_selftest_bounded_wait(limit_cycles: int, stream=None) -> int:
    return int(_lib.lca_selftest_bounded_wait(int(limit_cycles), _stream(stream)))


def lca_last_device_status(stream=None) -> int:
    return int(_lib.lca_last_device_status(_stream(stream)))


# ----------------------------------------------------------------------- allocation helpers
def make_params(variant: str, batch: int, seq_len: int, n_q_heads: int, n_kv_heads: int, d_sem: int,
                d_pos: int, group_size: int, window: int, softmax_scale: float,
                n_summary_q: int = 0, rep_logit_bias: float = 0.0) -> LcaParams:
    v = LCA_VARIANT_MLA if variant == "mla" else LCA_VARIANT_GQA
    return LcaParams(v, batch, seq_len, n_q_heads, n_kv_heads, d_sem, d_pos, group_size, window,
                     n_summary_q, softmax_scale, rep_logit_bias, 0, 0)


def params_from_config(cfg, batch: Optional[int] = None, **kw) -> LcaParams:
    d_pos = cfg.d_pos if cfg.variant == "mla" else cfg.d_sem
    p = make_params(cfg.variant, cfg.batch if batch is None else batch, cfg.seq_len, cfg.n_q_heads,
                    cfg.n_kv_heads, cfg.d_sem, d_pos, cfg.group_size, cfg.window, cfg.softmax_scale)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def _check(st: int, where: str):
    if st != LCA_OK:
        raise LcaError(st, where)


def workspace(params: LcaParams, which: int, device) -> Optional[torch.Tensor]:
    n = lca_workspace_bytes(params, which)
    return torch.empty(max(n, 16), dtype=torch.uint8, device=device)


def condense(params: LcaParams, q_tail_sem, q_tail_pos, kv_sem, kv_pos, qbar: Optional[torch.Tensor] = None,
             q_tail_batch_stride: Optional[int] = None, want_scores: bool = False, out=None, ws=None,
             stream=None):
    """Allocate the condensed cache and run lca_condense.  Returns dict(cache_sem, cache_pos,
    anchor_idx, scores, m, k)."""
    dev = kv_sem.device
    m, k = lca_partition(params)
    B, Hkv = params.batch, params.n_kv_heads
    if out is None:
        out = dict(cache_sem=torch.empty((B, m + k, Hkv, params.d_sem), dtype=torch.bfloat16, device=dev),
                   cache_pos=torch.empty((B, m + k, Hkv, params.d_pos), dtype=torch.bfloat16, device=dev),
                   anchor_idx=torch.empty((B, max(m, 1), Hkv), dtype=torch.int32, device=dev))
    scores = torch.empty((B, Hkv, max(m, 1) * params.group_size), dtype=torch.float64, device=dev) if want_scores else None
    if ws is None:
        ws = workspace(params, LCA_WS_CONDENSE, dev)
    n = params.n_summary_q if params.n_summary_q > 0 else params.group_size
    n = min(n, params.seq_len)
    stride = n if q_tail_batch_stride is None else q_tail_batch_stride
    st = lca_condense(params, q_tail_sem, q_tail_pos, stride, qbar, kv_sem, kv_pos, out["cache_sem"],
                      out["cache_pos"], out["anchor_idx"], scores, ws, stream=stream)
    _check(st, "lca_condense")
    res = dict(out)
    res.update(scores=scores, m=m, k=k, ws=ws)
    return res


def prefill_attention(params: LcaParams, q_sem, q_pos, kv_sem, kv_pos, cache_sem, cache_pos, out=None,
                      want_lse: bool = False, ws=None, stream=None):
    dev = kv_sem.device
    B, L, H = params.batch, params.seq_len, params.n_q_heads
    if out is None:
        out = torch.empty((B, L, H, params.d_sem), dtype=torch.bfloat16, device=dev)
    lse = torch.empty((B, L, H), dtype=torch.float32, device=dev) if want_lse else None
    if ws is None:
        ws = workspace(params, LCA_WS_PREFILL, dev)
    st = lca_prefill_attention(params, q_sem, q_pos, kv_sem, kv_pos, cache_sem, cache_pos, out, lse, ws,
                               stream=stream)
    _check(st, "lca_prefill_attention")
    return out, lse


def decode_attention(params: LcaParams, q_sem, q_pos, cache_sem, cache_pos, cache_rows, n_rep: int,
                     out=None, want_lse: bool = False, ws=None, stream=None):
    dev = cache_sem.device
    B, H = params.batch, params.n_q_heads
    cap = cache_sem.shape[1]
    if out is None:
        out = torch.empty((B, H, params.d_sem), dtype=torch.bfloat16, device=dev)
    lse = torch.empty((B, H), dtype=torch.float32, device=dev) if want_lse else None
    if ws is None:
        ws = workspace(params, LCA_WS_DECODE, dev)
    st = lca_decode_attention(params, q_sem, q_pos, cache_sem, cache_pos, cache_rows, cap, n_rep, out, lse,
                              ws, stream=stream)
    _check(st, "lca_decode_attention")
    return out, lse


def condense_varlen(params: LcaParams, seq_lens, q_sem, q_pos, kv_sem, kv_pos, qbar: Optional[torch.Tensor] = None,
                    stream=None):
    """Packed batch of sequences of different lengths: allocate the packed cache and run lca_condense_varlen.
    Returns dict(cache_sem, cache_pos, anchor_idx, token_offsets, cache_row_offsets, group_offsets)."""
    dev = kv_sem.device
    p = LcaParams.from_buffer_copy(params)
    p.batch, p.seq_len = len(seq_lens), max(seq_lens)
    tok, cache, grp = lca_varlen_layout(p, seq_lens)
    Hkv = p.n_kv_heads
    out = dict(cache_sem=torch.empty((cache[-1], Hkv, p.d_sem), dtype=torch.bfloat16, device=dev),
               cache_pos=torch.empty((cache[-1], Hkv, p.d_pos), dtype=torch.bfloat16, device=dev),
               anchor_idx=torch.empty((max(grp[-1], 1), Hkv), dtype=torch.int32, device=dev))
    ws = workspace(p, LCA_WS_CONDENSE_VARLEN, dev)
    st = lca_condense_varlen(p, seq_lens, q_sem, q_pos, qbar, kv_sem, kv_pos, out["cache_sem"], out["cache_pos"],
                             out["anchor_idx"], ws, stream=stream)
    _check(st, "lca_condense_varlen")
    out.update(token_offsets=tok, cache_row_offsets=cache, group_offsets=grp, ws=ws)
    return out


def prefill_attention_varlen(params: LcaParams, seq_lens, q_sem, q_pos, kv_sem, kv_pos, cache_sem, cache_pos,
                             want_lse: bool = False, stream=None):
    dev = kv_sem.device
    p = LcaParams.from_buffer_copy(params)
    p.batch, p.seq_len = len(seq_lens), max(seq_lens)
    T, H = sum(seq_lens), p.n_q_heads
    out = torch.empty((T, H, p.d_sem), dtype=torch.bfloat16, device=dev)
    lse = torch.empty((T, H), dtype=torch.float32, device=dev) if want_lse else None
    ws = workspace(p, LCA_WS_PREFILL_VARLEN, dev)
    st = lca_prefill_attention_varlen(p, seq_lens, q_sem, q_pos, kv_sem, kv_pos, cache_sem, cache_pos, out, lse, ws,
                                      stream=stream)
    _check(st, "lca_prefill_attention_varlen")
    return out, lse


def latent_to_value(attn_latent: torch.Tensor, w_uv: torch.Tensor, out=None, stream=None):
    """out_v[..., h, :] = attn_latent[..., h, :] @ w_uv[h]  (attn_latent [..., H, d_latent], w_uv [H, d_latent, d_v])."""
    H, d_latent, d_v = w_uv.shape
    n_tokens = attn_latent.numel() // (H * d_latent)
    if out is None:
        out = torch.empty(attn_latent.shape[:-1] + (d_v,), dtype=torch.bfloat16, device=attn_latent.device)
    _check(lca_latent_to_value(attn_latent, w_uv, out, n_tokens, H, d_latent, d_v, stream=stream), "lca_latent_to_value")
    return out


def decode_update(params: LcaParams, q_tail_sem, q_tail_pos, cache_sem, cache_pos, n_rep, cache_rows,
                  qbar: Optional[torch.Tensor] = None, ws=None, stream=None):
    """Run lca_decode_update in place on the cache buffers and counters; returns anchor offsets [B, Hkv]."""
    dev = cache_sem.device
    anchor = torch.empty((params.batch, params.n_kv_heads), dtype=torch.int32, device=dev)
    if ws is None:
        ws = workspace(params, LCA_WS_UPDATE, dev)
    n = params.n_summary_q if params.n_summary_q > 0 else params.group_size
    st = lca_decode_update(params, q_tail_sem, q_tail_pos, n, qbar, cache_sem, cache_pos, cache_sem.shape[1], n_rep,
                           cache_rows, anchor, ws, stream=stream)
    _check(st, "lca_decode_update")
    return anchor


def ring_from_packed(params: LcaParams, packed_sem, packed_pos, packed_rows, n_rep, ring_row_capacity: int, stream=None):
    """Allocate zeroed ring buffers and fill them from a packed cache.  Returns (ring_sem, ring_pos, n_tok [B] int32)."""
    dev = packed_sem.device
    B = params.batch
    ring_sem = torch.zeros((B, ring_row_capacity) + tuple(packed_sem.shape[2:]), dtype=torch.bfloat16, device=dev)
    ring_pos = torch.zeros((B, ring_row_capacity) + tuple(packed_pos.shape[2:]), dtype=torch.bfloat16, device=dev)
    n_tok = torch.empty((B,), dtype=torch.int32, device=dev)
    st = lca_ring_from_packed(params, packed_sem, packed_pos, packed_rows, n_rep, packed_sem.shape[1], ring_sem, ring_pos,
                              ring_row_capacity, n_tok, stream=stream)
    _check(st, "lca_ring_from_packed")
    return ring_sem, ring_pos, n_tok


def decode_attention_ring(params: LcaParams, q_sem, q_pos, ring_sem, ring_pos, n_rep, n_tok, out=None,
                          want_lse: bool = False, ws=None, stream=None):
    dev = ring_sem.device
    B, H = params.batch, params.n_q_heads
    if out is None:
        out = torch.empty((B, H, params.d_sem), dtype=torch.bfloat16, device=dev)
    lse = torch.empty((B, H), dtype=torch.float32, device=dev) if want_lse else None
    if ws is None:
        ws = workspace(params, LCA_WS_DECODE, dev)
    st = lca_decode_attention_ring(params, q_sem, q_pos, ring_sem, ring_pos, n_rep, n_tok, ring_sem.shape[1], out, lse,
                                   ws, stream=stream)
    _check(st, "lca_decode_attention_ring")
    return out, lse


def decode_update_ring(params: LcaParams, q_tail_sem, q_tail_pos, ring_sem, ring_pos, n_rep, n_tok,
                       qbar: Optional[torch.Tensor] = None, ws=None, stream=None):
    """Run lca_decode_update_ring in place on the ring buffers and n_rep; returns anchor offsets [B, Hkv]."""
    dev = ring_sem.device
    anchor = torch.empty((params.batch, params.n_kv_heads), dtype=torch.int32, device=dev)
    if ws is None:
        ws = workspace(params, LCA_WS_UPDATE, dev)
    n = params.n_summary_q if params.n_summary_q > 0 else params.group_size
    st = lca_decode_update_ring(params, q_tail_sem, q_tail_pos, n, qbar, ring_sem, ring_pos, ring_sem.shape[1], n_rep,
                                n_tok, anchor, ws, stream=stream)
    _check(st, "lca_decode_update_ring")
    return anchor


def decode_step_update_ring(params: LcaParams, q_sem, q_pos, qsum, qcount, ring_sem, ring_pos, n_rep, n_tok, ws=None,
                            anchor=None, stream=None):
    """Run lca_decode_step_update_ring in place (qsum [B, Hkv, dk] float64, qcount [B] int32); returns anchor offsets."""
    dev = ring_sem.device
    if anchor is None:
        anchor = torch.empty((params.batch, params.n_kv_heads), dtype=torch.int32, device=dev)
    if ws is None:
        ws = workspace(params, LCA_WS_UPDATE, dev)
    st = lca_decode_step_update_ring(params, q_sem, q_pos, qsum, qcount, ring_sem, ring_pos, ring_sem.shape[1], n_rep, n_tok,
                                     anchor, ws, stream=stream)
    _check(st, "lca_decode_step_update_ring")
    return anchor


def paged8_cache(pages_sem, pages_pos, scale_sem, scale_pos, block_table, page_size: Optional[int] = None,
                 n_pages: Optional[int] = None) -> LcaPaged8:
    """Descriptor of a paged 8-bit cache over the caller's tensors (any of them may be None for calls that do not use it):
    pages [n_pages, Hkv, page_size, d] of one byte per element (uint8 or float8_e4m3fn), scales [n_pages, Hkv] float32,
    block_table [batch, table_width] int32, all on one device.  ``page_update`` needs the table, page_size and n_pages only."""
    if pages_sem is not None:
        n_pages, page_size = pages_sem.shape[0], pages_sem.shape[2]
    tensors = (pages_sem, pages_pos, scale_sem, scale_pos, block_table)
    for t, want in ((pages_sem, 1), (pages_pos, 1), (scale_sem, 4), (scale_pos, 4), (block_table, 4)):
        if t is not None and (t.element_size() != want or (want == 4 and t.is_floating_point() == (t is block_table))):
            raise ValueError("pages hold one byte per element, scales are float32, block tables int32")
    if len({t.device for t in tensors if t is not None}) > 1:
        raise ValueError("the pages, scales and tables of a cache are on one device")
    if pages_pos is not None and (pages_sem is None or pages_pos.shape[:3] != pages_sem.shape[:3]):
        raise ValueError("both pools have the same pages: [n_pages, Hkv, page_size, d]")
    for t in (scale_sem, scale_pos):
        if t is not None and (pages_sem is None or t.shape != pages_sem.shape[:2]):
            raise ValueError("a scale for each page and KV head: [n_pages, Hkv]")
    if block_table is not None and block_table.dim() != 2:
        raise ValueError("block_table is [batch, table_width]")
    c = LcaPaged8(_ptr(pages_sem), _ptr(pages_pos), _ptr(scale_sem), _ptr(scale_pos), _ptr(block_table), int(n_pages or 0),
                  int(page_size or 0), 0 if block_table is None else block_table.shape[1])
    c.tensors = tensors
    c.device = next((t.get_device() for t in tensors if t is not None), None)
    c.batch = None if block_table is None else block_table.shape[0]
    if pages_sem is not None and pages_pos is not None:
        c.layout = (pages_sem.shape[1], pages_sem.shape[3], pages_pos.shape[3])
    return c


def new_paged8_cache(params: LcaParams, n_pages: int, page_size: int, table_width: int, device) -> LcaPaged8:
    """Allocate a pool of pages, its scales and empty block tables for params.batch sequences."""
    Hkv = params.n_kv_heads
    scale = torch.ones((n_pages, Hkv), dtype=torch.float32, device=device)
    return paged8_cache(torch.zeros((n_pages, Hkv, page_size, params.d_sem), dtype=torch.uint8, device=device),
                        torch.zeros((n_pages, Hkv, page_size, params.d_pos), dtype=torch.uint8, device=device), scale,
                        torch.ones_like(scale) if params.variant == LCA_VARIANT_GQA else None,
                        torch.full((params.batch, table_width), -1, dtype=torch.int32, device=device))


# The helpers below are called for every step of every layer: ctypes takes the structures as they are (the declared argument
# types make it pass their address), which costs half of what C.byref does.
_I32, _F32, _F64, _BF16 = torch.int32, torch.float32, torch.float64, torch.bfloat16


def _arg(x, dtype, n, dev):
    """Address of a dense tensor of this type with at least n elements on device dev; None stays None."""
    if x is None:
        return None
    if x.dtype is not dtype or x.get_device() != dev or x.numel() < n or not x.is_contiguous():
        raise ValueError(f"expected a dense {dtype} tensor of at least {n} elements on cuda:{dev}, not "
                         f"{x.dtype} {list(x.shape)} on {x.device}")
    return x.data_ptr()


def _queries(x, B, tokens, heads, d, dev):
    """Address of bf16 queries [B, tokens, heads, d].  More sequences may follow, but each has to have exactly these rows: the
    library finds a sequence by them."""
    if x is None:
        return None
    n = tokens * heads * d
    if x.shape[1:] != (tokens, heads, d) if x.dim() == 4 else x.numel() != B * n:
        raise ValueError(f"expected queries of {tokens} x {heads} x {d} for every sequence, not {list(x.shape)}")
    return _arg(x, _BF16, B * n, dev)


def _paged_device(params: LcaParams, cache, stream, table: bool = True):
    """The cache's device, which has to be the current one, the stream to launch on and (n_kv_heads, d_sem, d_pos); the
    tables and pages have to be those of params."""
    dev = cache.device
    if dev is None or dev < 0 or dev != torch.cuda.current_device():
        raise ValueError("the cache's tensors are not on the current CUDA device")
    if table and (cache.batch is None or cache.batch < params.batch):
        raise ValueError("block_table has a row for every sequence of params.batch")
    layout = (params.n_kv_heads, params.d_sem, params.d_pos)
    if cache.layout != layout and cache.layout is not None:
        raise ValueError(f"pages of (n_kv_heads, d_sem, d_pos) = {cache.layout} do not belong to these parameters")
    return dev, torch._C._cuda_getCurrentRawStream(dev) if stream is None else _stream(stream), layout


def _new(make, shape, dtype, device, stream):
    """A tensor for the caller made on the stream that its call runs on: its memory, and the fill, then come before the call."""
    if stream is None:
        return make(shape, dtype=dtype, device=device)
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(int(stream))
    with torch.cuda.stream(stream):
        return make(shape, dtype=dtype, device=device)


def page_update(params: LcaParams, cache, n_rep, n_tok, held_rep, held_tok, free_pages, n_free, slot_map, row_offsets,
                status, rows_per_seq: int = 0, stream=None):
    """Run lca_page_update in place on the tables (of an 8-bit or a 4-bit cache), the free list and the held state; returns
    slot_map.  `status` is a device tensor: read it where the caller has to know (0: done)."""
    dev, at, _ = _paged_device(params, cache, stream)
    if type(cache) is LcaPaged4:
        cache = cache.pages
    B = params.batch
    done, slots = _arg(status, _I32, 1, dev), _arg(slot_map, _I32, 0, dev)
    if slots == 0:                             # an empty tensor has no address, and no room for a row either: not "not wanted"
        slots = done
    _check(_lib.lca_page_update(params, cache, _arg(n_rep, _I32, B, dev), _arg(n_tok, _I32, B, dev),
                                _arg(held_rep, _I32, B, dev), _arg(held_tok, _I32, B, dev), _arg(free_pages, _I32, cache.n_pages, dev),
                                _arg(n_free, _I32, 1, dev), slots, 0 if slot_map is None else slot_map.numel(),
                                rows_per_seq, _arg(row_offsets, _I32, B + 1, dev), done, at), "lca_page_update")
    return slot_map


def paged8_write(params: LcaParams, cache: LcaPaged8, rows_sem, rows_pos, slot_map, stream=None):
    """Quantise rows into the pages that slot_map names (in place)."""
    dev, at, (Hkv, d_sem, d_pos) = _paged_device(params, cache, stream, table=False)
    n = slot_map.numel()
    _check(_lib.lca_paged8_write(params, cache, _arg(rows_sem, _BF16, n * Hkv * d_sem, dev),
                                 _arg(rows_pos, _BF16, n * Hkv * d_pos, dev), _arg(slot_map, _I32, n, dev), n, at), "lca_paged8_write")


def workspace_paged8(params: LcaParams, cache: LcaPaged8, q_len: int, device) -> torch.Tensor:
    return torch.empty(max(lca_paged8_workspace_bytes(params, cache, q_len), 16), dtype=torch.uint8, device=device)


def _decode_attention_paged(call, ws_bytes, name, params, cache, q_sem, q_pos, n_rep, n_tok, out, lse, want_lse, ws, stream):
    dev, at, (_, d_sem, d_pos) = _paged_device(params, cache, stream)
    B, q_len, H = params.batch, q_pos.shape[1], params.n_q_heads
    if out is None:
        out = _new(torch.empty, (B, q_len, H, d_sem), _BF16, q_pos.device, stream)
    if lse is None and want_lse:
        lse = _new(torch.empty, (B, q_len, H), _F32, q_pos.device, stream)
    if ws is None:
        ws = _new(torch.empty, max(ws_bytes(params, cache, q_len), 16), torch.uint8, q_pos.device, stream)
    rows = B * q_len * H
    _check(call(
        params, cache, _queries(q_sem, B, q_len, H, d_sem, dev), _queries(q_pos, B, q_len, H, d_pos, dev), q_len,
        _arg(n_rep, _I32, B, dev), _arg(n_tok, _I32, B, dev), _arg(out, _BF16, rows * d_sem, dev), _arg(lse, _F32, rows, dev),
        _arg(ws, torch.uint8, 0, dev), ws.numel(), at), name)
    return out, lse


def decode_attention_paged8(params: LcaParams, cache: LcaPaged8, q_sem, q_pos, n_rep, n_tok, out=None, lse=None,
                            want_lse: bool = False, ws=None, stream=None):
    """Attention of q_pos.shape[1] new tokens per sequence (q_pos [B, q_len, H, d_pos]) over the paged cache."""
    return _decode_attention_paged(_lib.lca_decode_attention_paged8, lca_paged8_workspace_bytes, "lca_decode_attention_paged8", params, cache,
                                   q_sem, q_pos, n_rep, n_tok, out, lse, want_lse, ws, stream)


def _decode_update_paged(call, name, params, cache, q_tail_sem, q_tail_pos, n_rep, n_tok, n_rep_new, rep_sem, rep_pos, qbar, anchor, ws, stream):
    dev, at, (Hkv, d_sem, d_pos) = _paged_device(params, cache, stream)
    B = params.batch
    if n_rep_new is None:
        n_rep_new = _new(torch.empty, (B,), _I32, n_tok.device, stream)
    if rep_sem is None:
        rep_sem = _new(torch.zeros, (B, Hkv, d_sem), _BF16, n_tok.device, stream)
    if rep_pos is None:
        rep_pos = _new(torch.zeros, (B, Hkv, d_pos), _BF16, n_tok.device, stream)
    if anchor is None:
        anchor = _new(torch.empty, (B, Hkv), _I32, n_tok.device, stream)
    if ws is None:
        ws = _new(torch.empty, max(lca_workspace_bytes(params, LCA_WS_UPDATE), 16), torch.uint8, n_tok.device, stream)
    n = params.n_summary_q if params.n_summary_q > 0 else params.group_size
    H, blocks = params.n_q_heads, B * Hkv
    dk = d_pos + (d_sem if params.variant == LCA_VARIANT_MLA else 0)
    _check(call(
        params, cache, _queries(q_tail_sem, B, n, H, d_sem, dev), _queries(q_tail_pos, B, n, H, d_pos, dev), n,
        _arg(qbar, _F32, blocks * dk, dev), _arg(n_rep, _I32, B, dev), _arg(n_tok, _I32, B, dev), _arg(n_rep_new, _I32, B, dev),
        _arg(rep_sem, _BF16, blocks * d_sem, dev), _arg(rep_pos, _BF16, blocks * d_pos, dev), _arg(anchor, _I32, blocks, dev),
        _arg(ws, torch.uint8, 0, dev), ws.numel(), at), name)
    return n_rep_new, rep_sem, rep_pos, anchor


def decode_update_paged8(params: LcaParams, cache: LcaPaged8, q_tail_sem, q_tail_pos, n_rep, n_tok, n_rep_new=None, rep_sem=None,
                         rep_pos=None, qbar: Optional[torch.Tensor] = None, anchor=None, ws=None, stream=None):
    """Run lca_decode_update_paged8 (q_tail_* [B, n, H, d], exactly the n latest positions, n = n_summary_q or group_size, or the
    ready summary query qbar [B, Hkv, dk]); returns (n_rep_new [B], rep_sem [B, Hkv, d_sem], rep_pos [B, Hkv, d_pos], anchor [B, Hkv])."""
    return _decode_update_paged(_lib.lca_decode_update_paged8, "lca_decode_update_paged8", params, cache, q_tail_sem, q_tail_pos, n_rep, n_tok,
                                n_rep_new, rep_sem, rep_pos, qbar, anchor, ws, stream)


def paged4_cache(pages_sem, pages_pos, shift_sem, shift_pos, exp_sem, exp_pos, block_table) -> LcaPaged4:
    """Descriptor of a paged 4-bit cache over the caller's tensors: pages [n_pages, Hkv, page_size, d / 2], shifts [n_pages, Hkv,
    page_size, d / 64] and exponents [n_pages, Hkv, page_size] (exp_pos None for MLA), all of one byte per element, block_table
    [batch, table_width] int32 (None for calls that do not use it), all on one device."""
    if pages_sem is None or pages_pos is None or pages_sem.dim() != 4 or pages_pos.shape[:3] != pages_sem.shape[:3]:
        raise ValueError("both pools have the same pages: [n_pages, Hkv, page_size, d / 2]")
    tensors = (pages_sem, pages_pos, shift_sem, shift_pos, exp_sem, exp_pos, block_table)
    n_pages, Hkv, page_size = pages_sem.shape[:3]
    for t, pool in ((shift_sem, pages_sem), (shift_pos, pages_pos)):
        if t is None or t.shape != pool.shape[:3] + (pool.shape[3] // 32,):
            raise ValueError("half a byte for each 32 columns of a row: shifts [n_pages, Hkv, page_size, d / 64]")
    if exp_sem is None or any(t is not None and t.shape != pages_sem.shape[:3] for t in (exp_sem, exp_pos)):
        raise ValueError("an exponent for each row and KV head: [n_pages, Hkv, page_size]")
    if any(t is not None and t.element_size() != 1 for t in tensors[:6]):
        raise ValueError("pages, shifts and exponents hold one byte per element")
    if block_table is not None and (block_table.dim() != 2 or block_table.dtype is not torch.int32):
        raise ValueError("block_table is [batch, table_width] int32")
    if len({t.device for t in tensors if t is not None}) > 1:
        raise ValueError("the pages, scales and tables of a cache are on one device")
    width = 0 if block_table is None else block_table.shape[1]
    c = LcaPaged4(*(_ptr(t) for t in tensors), n_pages, page_size, width)
    c.tensors = tensors
    c.device = pages_sem.get_device()
    c.batch = None if block_table is None else block_table.shape[0]
    c.layout = (Hkv, 2 * pages_sem.shape[3], 2 * pages_pos.shape[3])
    c.pages = LcaPaged8(None, None, None, None, _ptr(block_table), n_pages, page_size, width)
    return c


def new_paged4_cache(params: LcaParams, n_pages: int, page_size: int, table_width: int, device) -> LcaPaged4:
    """Allocate a pool of pages and empty block tables for params.batch sequences."""
    row = (n_pages, params.n_kv_heads, page_size)
    new = lambda *d: torch.zeros(row + d, dtype=torch.uint8, device=device)  # noqa: E731
    return paged4_cache(new(params.d_sem // 2), new(params.d_pos // 2), new(params.d_sem // 64), new(params.d_pos // 64), new(),
                        new() if params.variant == LCA_VARIANT_GQA else None,
                        torch.full((params.batch, table_width), -1, dtype=torch.int32, device=device))


def paged4_write(params: LcaParams, cache: LcaPaged4, rows_sem, rows_pos, slot_map, stream=None):
    """Quantise rows into the slots that slot_map names (in place)."""
    dev, at, (Hkv, d_sem, d_pos) = _paged_device(params, cache, stream, table=False)
    n = slot_map.numel()
    _check(_lib.lca_paged4_write(params, cache, _arg(rows_sem, _BF16, n * Hkv * d_sem, dev),
                                 _arg(rows_pos, _BF16, n * Hkv * d_pos, dev), _arg(slot_map, _I32, n, dev), n, at), "lca_paged4_write")


def paged4_read(params: LcaParams, cache: LcaPaged4, slot_map, rows_sem=None, rows_pos=None, stream=None):
    """The values of the rows that slot_map names: (rows_sem [n, Hkv, d_sem], rows_pos [n, Hkv, d_pos]) bf16.  Rows of a slot
    outside the pool are left as they are, zero where this call makes the tensor."""
    dev, at, (Hkv, d_sem, d_pos) = _paged_device(params, cache, stream, table=False)
    n = slot_map.numel()
    if rows_sem is None:
        rows_sem = _new(torch.zeros, (n, Hkv, d_sem), _BF16, slot_map.device, stream)
    if rows_pos is None:
        rows_pos = _new(torch.zeros, (n, Hkv, d_pos), _BF16, slot_map.device, stream)
    _check(_lib.lca_paged4_read(params, cache, _arg(rows_sem, _BF16, n * Hkv * d_sem, dev), _arg(rows_pos, _BF16, n * Hkv * d_pos, dev),
                                _arg(slot_map, _I32, n, dev), n, at), "lca_paged4_read")
    return rows_sem, rows_pos


def workspace_paged4(params: LcaParams, cache: LcaPaged4, q_len: int, device) -> torch.Tensor:
    return torch.empty(max(lca_paged4_workspace_bytes(params, cache, q_len), 16), dtype=torch.uint8, device=device)


def decode_attention_paged4(params: LcaParams, cache: LcaPaged4, q_sem, q_pos, n_rep, n_tok, out=None, lse=None,
                            want_lse: bool = False, ws=None, stream=None):
    """Attention of q_pos.shape[1] new tokens per sequence (q_pos [B, q_len, H, d_pos]) over the paged cache."""
    return _decode_attention_paged(_lib.lca_decode_attention_paged4, lca_paged4_workspace_bytes, "lca_decode_attention_paged4", params, cache,
                                   q_sem, q_pos, n_rep, n_tok, out, lse, want_lse, ws, stream)


def decode_update_paged4(params: LcaParams, cache: LcaPaged4, q_tail_sem, q_tail_pos, n_rep, n_tok, n_rep_new=None, rep_sem=None,
                         rep_pos=None, qbar: Optional[torch.Tensor] = None, anchor=None, ws=None, stream=None):
    """Run lca_decode_update_paged4; arguments and results as for decode_update_paged8."""
    return _decode_update_paged(_lib.lca_decode_update_paged4, "lca_decode_update_paged4", params, cache, q_tail_sem, q_tail_pos, n_rep, n_tok,
                                n_rep_new, rep_sem, rep_pos, qbar, anchor, ws, stream)


# ------------------------------------------------------------------------------------------- around a speculative step
def _device(x, where: str):
    """Index of the CUDA device of a tensor, which has to be the current one."""
    dev = x.get_device()
    if dev < 0 or dev != torch.cuda.current_device():
        raise ValueError(f"{where} takes tensors on the current CUDA device, not on {x.device}")
    return dev


def _raw_stream(dev, stream):
    return torch._C._cuda_getCurrentRawStream(dev) if stream is None else _stream(stream)


def rope_frequencies(rot_dim: int, base: float = 10000.0, kind: int = ROPE_PLAIN, scale: float = 1.0, trained_len: float = 0.0,
                     fast: float = 32.0, slow: float = 1.0, device="cuda"):
    """(freqs [rot_dim / 2] float64 on `device`, factor): the frequencies of lca_rope_frequencies, which `rope` takes."""
    f, factor = (C.c_double * max(int(rot_dim) // 2, 1))(), C.c_float()
    _check(lca_rope_frequencies(kind, rot_dim, base, scale, trained_len, fast, slow, f, factor), "lca_rope_frequencies")
    return torch.tensor(list(f), dtype=torch.float64, device=device), factor.value


_ROPE_TYPES = {torch.bfloat16: LCA_DTYPE_BF16, torch.float32: LCA_DTYPE_FP32}


def _heads(v, T, d, dtype, dev):
    """(heads, address, token stride, head stride) of a tensor [T, heads, d] whose columns lie side by side."""
    shape, strides = v.shape, v.stride()
    if len(shape) != 3 or shape[0] != T or shape[2] != d or (strides[2] != 1 and d > 1) or v.dtype is not dtype or v.get_device() != dev:
        raise ValueError(f"expected [T, heads, {d}] of {dtype} on cuda:{dev} with neighbouring columns, T = {T}, not "
                         f"{v.dtype} {list(shape)} with strides {list(strides)} on {v.device}")
    return shape[1], v.data_ptr(), strides[0], strides[1]


def rope(q, k, positions, freqs, interleaved: bool = False, inverse: bool = False, factor: float = 1.0, q_out=None, k_out=None, stream=None):
    """Rotate q [T, heads, d] and k [T, kv_heads, d] (either may be None) by the angles positions [T] int32 times freqs [rot / 2]
    float64: columns 0 .. rot - 1 of every head, the others are copied.  The tensors may be views (slices of a projection) as long
    as the columns of a head lie side by side; q_out may be q and k_out may be k, otherwise outputs overlap nothing.  Returns (q_out, k_out)."""
    x = q if q is not None else k
    if x is None:
        raise ValueError("rope takes queries, keys or both")
    T, _, d = x.shape
    dtype, dev = x.dtype, _device(x, "rope")
    code = _ROPE_TYPES.get(dtype)
    if code is None:
        raise ValueError(f"rope takes bfloat16 or float32, not {dtype}")
    parts, outs = [], []
    for t, o in ((q, q_out), (k, k_out)):
        if t is None:
            parts.append((0,) + 6 * (None,))
            outs.append(None)
            continue
        if o is None:
            o = _new(torch.empty, tuple(t.shape), dtype, t.device, stream)
        n, at, st, sh = _heads(t, T, d, dtype, dev)
        m, to, ot, oh = _heads(o, T, d, dtype, dev)
        if m != n or (ot == 0 and T > 1) or (oh == 0 and n > 1):
            raise ValueError("an output has the heads of its input, each at a place of its own")
        parts.append((n, at, st, sh, to, ot, oh))
        outs.append(o)
    (nq, a, b, c, e, f, g), (nk, h, i, j, l, m, n) = parts
    args = LcaRopeArgs(code, interleaved, inverse, nq, nk, d, 2 * freqs.numel(), factor, T, _arg(positions, _I32, T, dev), _arg(freqs, _F64, 1, dev),
                       a, b or 0, c or 0, e, f or 0, g or 0, h, i or 0, j or 0, l, m or 0, n or 0)
    if T > 0:
        _check(_lib.lca_rope(args, _raw_stream(dev, stream)), "lca_rope")
    return outs[0], outs[1]


def verify_drafts(target_probs, draft_probs, draft_tokens, u_accept, u_sample, n_draft=None, n_tok=None, accepted=None, out=None,
                  n_tok_out=None, stream=None):
    """Run lca_verify_drafts on target_probs [B, n + 1, V], draft_probs [B, n, V] (None: a drafter that is certain) of float32 or
    bfloat16, draft_tokens [B, n] int32, u_accept [B, n] and u_sample [B] float32.  Returns (accepted [B], tokens [B, n + 1],
    n_tok_out [B] or None) int32."""
    B, n1, V = target_probs.shape
    n = n1 - 1
    dev = _device(target_probs, "verify_drafts")
    dt = target_probs.dtype
    code = _ROPE_TYPES.get(dt)
    if code is None:
        raise ValueError(f"probabilities are float32 or bfloat16, not {dt}")
    if draft_probs is not None and draft_probs.shape != (B, n, V):
        raise ValueError(f"draft_probs is {[B, n, V]}, not {list(draft_probs.shape)}")
    for x, m in ((draft_tokens, n), (u_accept, n), (out, n1)):                 # the library finds a request by the length of these rows
        if x is not None and m > 0 and (x.shape[1] != m if x.dim() == 2 else x.numel() != B * m):
            raise ValueError(f"expected {m} elements for each of {B} requests, not {list(x.shape)}")
    if n_tok is None and n_tok_out is not None:
        raise ValueError("n_tok_out is n_tok less the rejected drafts: n_tok is missing")
    if accepted is None:
        accepted = _new(torch.empty, (B,), _I32, target_probs.device, stream)
    if out is None:
        out = _new(torch.empty, (B, n1), _I32, target_probs.device, stream)
    if n_tok is not None and n_tok_out is None:
        n_tok_out = _new(torch.empty, (B,), _I32, target_probs.device, stream)
    a = LcaVerifyArgs(code, B, n, V, _arg(target_probs, dt, B * n1 * V, dev), _arg(draft_probs, dt, B * n * V, dev),
                      _arg(draft_tokens, _I32, B * n, dev), _arg(n_draft, _I32, B, dev), _arg(u_accept, _F32, B * n, dev),
                      _arg(u_sample, _F32, B, dev), _arg(n_tok, _I32, B, dev), _arg(accepted, _I32, B, dev), _arg(out, _I32, B * n1, dev),
                      _arg(n_tok_out, _I32, B, dev))
    _check(_lib.lca_verify_drafts(a, _raw_stream(dev, stream)), "lca_verify_drafts")
    return accepted, out, n_tok_out
