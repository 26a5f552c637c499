"""ctypes binding of libspot (include/spot.h).

The functions ``spot_*`` mirror the C ABI one to one: they take torch tensors
(device memory), check dtype / device / contiguity / size, and pass raw
pointers plus the current HIP stream.  Every step of the path runs in the HIP
kernels of libspot.so; there is no fallback: if the library cannot be loaded
on a machine with a GPU, the first call raises.

The checks and the call itself run in a native module (csrc/binding.cpp) for
plain arguments; whatever it does not take (it answers None and has enqueued
nothing) goes through the Python checks below, which are the reference for
what is accepted and for every error.

Convenience wrappers without the ``spot_`` prefix allocate outputs with torch, on the
stream that the call goes to.
"""
from __future__ import annotations

import contextlib
import ctypes
import math
import os
import sys
import threading
from typing import Optional

import torch

from . import build as _build

SPOT_OK = 0
STATUS = {0: "ok", 1: "null pointer", 2: "invalid shape", 3: "unsupported", 4: "invalid rule",
          5: "workspace", 6: "HIP launch error", 7: "fused-step wait expired"}
SPOT_ERR_EXPIRED = 7
KFMT = {"bf16": 0, "int4": 1, "mxfp4": 2, "int8": 3, "mxfp8": 4}
BLK = 64

SYMBOLS = ["spot_status_str", "spot_version", "spot_selector_score",
           "spot_selector_score_q", "spot_selector_score_tokens",
           "spot_selector_score_tokens_blk", "spot_selector_project",
           "spot_selector_project_pooled", "spot_selector_pool",
           "spot_select_blocks",
           "spot_decode_workspace_bytes", "spot_sparse_decode", "spot_sparse_decode_blk",
           "spot_dense_decode",
           "spot_sparse_prefill", "spot_decode_step_workspace_bytes", "spot_decode_step",
           "spot_decode_step_q", "spot_decode_step_static", "spot_decode_step_status",
           "spot_test_force_expiry",
           "spot_rope_frequencies", "spot_rotary", "spot_rotary_append",
           "spot_paged_workspace_bytes", "spot_paged_attend", "spot_paged_weights",
           "spot_cache_evict", "spot_rotary_axes", "spot_rotary_append8",
           "spot_paged_attend_sinks", "spot_paged_attend8",
           "spot_probe_stream_read", "spot_probe_sink_words"]


class SpotError(RuntimeError):
    def __init__(self, fn: str, status: int):
        super().__init__(f"{fn} failed: status {status} ({STATUS.get(status, '?')})")
        self.status = status


_lock = threading.Lock()
_lib = None
_native = None     # csrc/binding.cpp, once the library is loaded


def load(path: Optional[str] = None):
    """Load libspot.so, building it first only if it does not exist."""
    global _lib
    with _lock:
        if _lib is not None and path is None:
            return _lib
        so = path or _build.SO
        if not os.path.exists(so):
            _build.build()
        elif path is None and _build.stale():
            print(f"warning: {so} is older than its sources; rebuild with "
                  "`python -m paper_2606_22874_amd.build`", file=sys.stderr)
        L = ctypes.CDLL(so)
        P, I, F, Z = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
        Q, D = ctypes.c_int64, ctypes.c_double
        L.spot_status_str.argtypes = [I]
        L.spot_status_str.restype = ctypes.c_char_p
        L.spot_version.restype = ctypes.c_char_p
        L.spot_selector_score.argtypes = [P, P, P, P, I, I, I, I, I, I, P, P, P]
        L.spot_selector_score_tokens.argtypes = [P, P, P, P, I, I, I, I, I, I, P, P, P]
        L.spot_selector_score_tokens_blk.argtypes = [P, P, P, P, I, I, I, I, I, I, I, P, P, P]
        L.spot_selector_score_q.argtypes = [P, P, I, P, P, P, I, I, I, I, I, I, P, P, P]
        L.spot_selector_project.argtypes = [P, P, P, P, P, I, I, I, I, I, F, P, P, P, I, I, P]
        L.spot_selector_pool.argtypes = [P, P, I, I, I, I, P, P, I, P]
        L.spot_selector_project_pooled.argtypes = [P, P, P, P, P, P, I, I, I, I, I, F, P, P, P,
                                                   P, I, P]
        L.spot_select_blocks.argtypes = [P, I, I, P, F, I, I, I, I, P, P, P, P]
        L.spot_decode_workspace_bytes.argtypes = [I, I, I, I, I]
        L.spot_decode_workspace_bytes.restype = Z
        L.spot_sparse_decode.argtypes = [P, P, P, P, P, P, I, I, I, I, I, I, F, P, P, P, Z, P]
        L.spot_sparse_decode_blk.argtypes = [P, P, P, P, P, P, I, I, I, I, I, I, I, F, P, P, P,
                                             Z, P]
        L.spot_dense_decode.argtypes = [P, P, P, P, I, I, I, I, I, F, P, P, P, Z, P]
        L.spot_sparse_prefill.argtypes = [P, P, P, I, P, P, I, I, I, I, I, F, P, P, P]
        L.spot_decode_step_workspace_bytes.argtypes = [I, I, I, I, I]
        L.spot_decode_step_workspace_bytes.restype = Z
        L.spot_decode_step.argtypes = [P, P, P, P, I, I, I, P, F, I, I, I, I, P, P, P, P, I, I,
                                       I, I, I, F, P, P, P, P, P, P, P, Z, P]
        L.spot_decode_step_q.argtypes = [P, P, I, P, P, P, I, I, I, P, F, I, I, I, I, P, P, P, P,
                                         I, I, I, I, I, F, P, P, P, P, P, P, P, Z, P]
        L.spot_decode_step_static.argtypes = [P, P, P, P, I, I, I, P, F, I, I, I, I, P, P, P, P,
                                              I, I, I, I, I, F, P, P, P, P, P, P, P]
        L.spot_decode_step_status.argtypes = [P, Z, I, I, I, I, I, P]
        L.spot_test_force_expiry.argtypes = [I]
        L.spot_test_force_expiry.restype = None
        L.spot_rope_frequencies.argtypes = [I, D, I, D, I, D, D, P]
        L.spot_rotary.argtypes = [P, Q, P, I, I, I, I, P, F, I, I, P, Q, P]
        L.spot_rotary_append.argtypes = [P, Q, P, Q, P, Q, I, P, P, I, I, I, P, P, I, I, I, I, I, I,
                                         P, F, I, P, P, P, P]
        L.spot_paged_workspace_bytes.argtypes = [I, I, I, I, I]
        L.spot_paged_workspace_bytes.restype = Z
        L.spot_paged_attend.argtypes = [P, I, P, P, P, I, I, I, P, P, I, I, I, I, I, F, F, P, I, P,
                                        P, P, P, P, Z, P]
        L.spot_paged_weights.argtypes = [P, P, I, P, P, I, I, I, P, P, I, I, I, I, I, F, F, P, I,
                                         P, P, P, F, P, P]
        L.spot_cache_evict.argtypes = [P, P, P, P, I, I, I, P, I, I, I, I, I, I, P, P, P, I, I, P,
                                       P, P, I, P]
        L.spot_rotary_axes.argtypes = [P, Q, P, I, P, I, I, I, I, P, F, I, I, P, Q, P]
        L.spot_rotary_append8.argtypes = [P, Q, P, Q, P, Q, I, P, I, P, P, I, I, I, P, P, I, I, I,
                                          I, I, I, P, F, I, P, P, P, P, P, P]
        L.spot_paged_attend_sinks.argtypes = [P, I, P, P, P, I, I, I, P, P, I, I, I, I, I, F, F, P,
                                              I, I, P, P, P, P, P, Z, P]
        L.spot_paged_attend8.argtypes = [P, I, P, P, P, P, P, I, I, I, P, P, I, I, I, I, I, F, F, P,
                                         I, I, P, P, P, P, P, Z, P]
        L.spot_probe_stream_read.argtypes = [P, Z, P, P]
        L.spot_probe_stream_read.restype = ctypes.c_int32
        L.spot_probe_sink_words.restype = I
        for name in ("spot_selector_score", "spot_selector_score_q", "spot_selector_score_tokens",
                     "spot_selector_score_tokens_blk",
                     "spot_selector_project", "spot_selector_project_pooled",
                     "spot_selector_pool", "spot_select_blocks", "spot_sparse_decode",
                     "spot_sparse_decode_blk",
                     "spot_dense_decode", "spot_sparse_prefill", "spot_decode_step",
                     "spot_decode_step_q", "spot_decode_step_static", "spot_decode_step_status",
                     "spot_rope_frequencies", "spot_rotary", "spot_rotary_append",
                     "spot_paged_attend", "spot_paged_weights", "spot_cache_evict",
                     "spot_rotary_axes", "spot_rotary_append8", "spot_paged_attend_sinks",
                     "spot_paged_attend8"):
            getattr(L, name).restype = ctypes.c_int32
        if path is None:
            _load_native(L)
            _lib = L
        return L


def _load_native(L):
    """Hands the library's entry points to the native marshalling module.  Where
    there is none for this torch and none can be built (no compiler or headers),
    every call takes the Python path, which does all of it, more slowly."""
    global _native
    try:
        if not _build.binding_fits():
            _build.build_binding()
        from . import _binding
        order = (L.spot_selector_score, L.spot_selector_score_q, L.spot_selector_score_tokens_blk,
                 L.spot_selector_project, L.spot_selector_project_pooled, L.spot_selector_pool,
                 L.spot_select_blocks, L.spot_sparse_decode_blk, L.spot_dense_decode,
                 L.spot_sparse_prefill, L.spot_decode_step, L.spot_decode_step_q,
                 L.spot_decode_step_static, L.spot_rotary, L.spot_rotary_append,
                 L.spot_paged_attend, L.spot_paged_weights, L.spot_cache_evict, L.spot_rotary_axes,
                 L.spot_rotary_append8, L.spot_paged_attend_sinks, L.spot_paged_attend8)
        _binding.init(tuple(ctypes.cast(f, ctypes.c_void_p).value for f in order),
                      torch.cuda.Stream)
        _native = _binding
    except (ImportError, OSError, RuntimeError) as e:
        print(f"warning: calls are marshalled in Python (10 us more each): {e}",
              file=sys.stderr)


# ------------------------------------------------------------- marshalling
def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    return ctypes.c_void_p(t.data_ptr())


def _stream(stream) -> ctypes.c_void_p:
    if stream is None:
        stream = torch.cuda.current_stream()
    if isinstance(stream, torch.cuda.Stream):
        return ctypes.c_void_p(stream.cuda_stream)
    return ctypes.c_void_p(int(stream))


def _dev(t: torch.Tensor, name: str, dtypes, numel: Optional[int] = None):
    if t is None:
        raise ValueError(f"{name} is required")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if t.data_ptr() % 16:
        raise ValueError(f"{name} must start on a 16-byte boundary")
    if dtypes is not None and t.dtype not in dtypes:
        raise ValueError(f"{name}: dtype {t.dtype} not in {dtypes}")
    if numel is not None and t.numel() < numel:
        raise ValueError(f"{name}: {t.numel()} elements, need {numel}")
    return t


BF16 = (torch.bfloat16, torch.int16)
I32 = (torch.int32,)
F32 = (torch.float32,)
U8 = (torch.uint8,)
CODES8 = (torch.uint8, torch.float8_e4m3fn)
SCALES8 = (torch.uint8, torch.float8_e8m0fnu)


PAGED_DTYPE = {torch.bfloat16: 0, torch.float16: 1}
ROPE_SCALING = {"none": 0, "linear": 1, "ntk": 2, "parts": 3, "yarn": 3}
ROPE_INTERLEAVED, ROPE_INVERSE = 1, 2
PAGED_WORKSPACE_ZEROS = 4096


def _check(fn: str, st: int):
    if st != SPOT_OK:
        raise SpotError(fn, st)


def _sel_cache(k, k_scale, f, n_keys, h_s, d_s, name, scale_name="k_scale"):
    """Checks n_keys selector keys (or queries) of h_s * d_s elements in format f."""
    if f == 0:
        _dev(k, name, BF16, n_keys * h_s * d_s)
        return
    per = h_s * d_s if f in (3, 4) else h_s * d_s // 2      # 8-bit or 4-bit codes
    _dev(k, name, U8 + (torch.int8,), n_keys * per)
    _dev(k_scale, scale_name, (torch.float16, torch.int16) if f in (1, 3) else U8,
         n_keys * h_s * d_s // 32)


# ------------------------------------------------------------- C ABI calls
def spot_selector_score(q_sel, w, k_sel, k_scale, kfmt, n_seq, rows_per_seq, nblk, h_s, d_s,
                        n_valid, scores, stream=None):
    if _native is not None:
        st = _native.selector_score(q_sel, w, k_sel, k_scale, kfmt, n_seq, rows_per_seq, nblk,
                                    h_s, d_s, n_valid, scores, stream)
        if st is not None:
            return _check("spot_selector_score", st)
    rows = n_seq * rows_per_seq
    f = KFMT[kfmt] if isinstance(kfmt, str) else int(kfmt)
    _dev(q_sel, "q_sel", BF16, rows * h_s * d_s)
    _dev(w, "w", F32, rows * h_s)
    _sel_cache(k_sel, k_scale, f, n_seq * nblk, h_s, d_s, "k_sel")
    if n_valid is not None:
        _dev(n_valid, "n_valid", I32, rows)
    _dev(scores, "scores", F32, rows * nblk)
    _check("spot_selector_score", load().spot_selector_score(
        _ptr(q_sel), _ptr(w), _ptr(k_sel), _ptr(k_scale), f, n_seq, rows_per_seq, nblk, h_s,
        d_s, _ptr(n_valid), _ptr(scores), _stream(stream)))


def spot_selector_score_q(q_sel, q_scale, qfmt, w, k_sel, k_scale, kfmt, n_seq, rows_per_seq,
                          nblk, h_s, d_s, n_valid, scores, stream=None):
    if _native is not None:
        st = _native.selector_score_q(q_sel, q_scale, qfmt, w, k_sel, k_scale, kfmt, n_seq,
                                      rows_per_seq, nblk, h_s, d_s, n_valid, scores, stream)
        if st is not None:
            return _check("spot_selector_score_q", st)
    rows = n_seq * rows_per_seq
    qf = KFMT[qfmt] if isinstance(qfmt, str) else int(qfmt)
    f = KFMT[kfmt] if isinstance(kfmt, str) else int(kfmt)
    _sel_cache(q_sel, q_scale, qf, rows, h_s, d_s, "q_sel", "q_scale")
    _dev(w, "w", F32, rows * h_s)
    _sel_cache(k_sel, k_scale, f, n_seq * nblk, h_s, d_s, "k_sel")
    if n_valid is not None:
        _dev(n_valid, "n_valid", I32, rows)
    _dev(scores, "scores", F32, rows * nblk)
    _check("spot_selector_score_q", load().spot_selector_score_q(
        _ptr(q_sel), _ptr(q_scale), qf, _ptr(w), _ptr(k_sel), _ptr(k_scale), f, n_seq,
        rows_per_seq, nblk, h_s, d_s, _ptr(n_valid), _ptr(scores), _stream(stream)))


def _tokens_args(q_sel, w, k_tok, k_scale, kfmt, n_seq, rows_per_seq, l_cap, blk, h_s, d_s,
                 seq_len, scores):
    rows = n_seq * rows_per_seq
    f = KFMT[kfmt] if isinstance(kfmt, str) else int(kfmt)
    _dev(q_sel, "q_sel", BF16, rows * h_s * d_s)
    _dev(w, "w", F32, rows * h_s)
    _sel_cache(k_tok, k_scale, f, n_seq * l_cap, h_s, d_s, "k_tok")
    if seq_len is not None:
        _dev(seq_len, "seq_len", I32, rows)
    _dev(scores, "scores", F32, rows * (l_cap // blk))
    return f


def spot_selector_score_tokens(q_sel, w, k_tok, k_scale, kfmt, n_seq, rows_per_seq, l_cap, h_s,
                               d_s, seq_len, scores, stream=None):
    if _native is not None:
        st = _native.selector_score_tokens_blk(q_sel, w, k_tok, k_scale, kfmt, n_seq,
                                               rows_per_seq, l_cap, BLK, h_s, d_s, seq_len,
                                               scores, stream)
        if st is not None:
            return _check("spot_selector_score_tokens", st)
    f = _tokens_args(q_sel, w, k_tok, k_scale, kfmt, n_seq, rows_per_seq, l_cap, 64, h_s, d_s,
                     seq_len, scores)
    _check("spot_selector_score_tokens", load().spot_selector_score_tokens(
        _ptr(q_sel), _ptr(w), _ptr(k_tok), _ptr(k_scale), f, n_seq, rows_per_seq, l_cap, h_s,
        d_s, _ptr(seq_len), _ptr(scores), _stream(stream)))


def spot_selector_score_tokens_blk(q_sel, w, k_tok, k_scale, kfmt, n_seq, rows_per_seq, l_cap,
                                   blk, h_s, d_s, seq_len, scores, stream=None):
    if _native is not None:
        st = _native.selector_score_tokens_blk(q_sel, w, k_tok, k_scale, kfmt, n_seq,
                                               rows_per_seq, l_cap, blk, h_s, d_s, seq_len,
                                               scores, stream)
        if st is not None:
            return _check("spot_selector_score_tokens_blk", st)
    f = _tokens_args(q_sel, w, k_tok, k_scale, kfmt, n_seq, rows_per_seq, l_cap, blk, h_s, d_s,
                     seq_len, scores)
    _check("spot_selector_score_tokens_blk", load().spot_selector_score_tokens_blk(
        _ptr(q_sel), _ptr(w), _ptr(k_tok), _ptr(k_scale), f, n_seq, rows_per_seq, l_cap, blk,
        h_s, d_s, _ptr(seq_len), _ptr(scores), _stream(stream)))


def spot_selector_project(h, w_q, w_k, w_w, pos, rows, d_model, h_s, d_s, rope_dim, rope_base,
                          q_out, w_out, k_cache, rows_per_seq, l_cap, stream=None):
    if _native is not None:
        st = _native.selector_project(h, w_q, w_k, w_w, pos, rows, d_model, h_s, d_s, rope_dim,
                                      rope_base, q_out, w_out, k_cache, rows_per_seq, l_cap,
                                      stream)
        if st is not None:
            return _check("spot_selector_project", st)
    n_out = h_s * d_s
    _dev(h, "h", BF16, rows * d_model)
    _dev(w_q, "w_q", BF16, n_out * d_model)
    _dev(w_k, "w_k", BF16, n_out * d_model)
    _dev(w_w, "w_w", BF16, h_s * d_model)
    _dev(pos, "pos", I32, rows)
    _dev(q_out, "q_out", BF16, rows * n_out)
    _dev(w_out, "w_out", F32, rows * h_s)
    _dev(k_cache, "k_cache", BF16, (rows // max(rows_per_seq, 1)) * l_cap * n_out)
    _check("spot_selector_project", load().spot_selector_project(
        _ptr(h), _ptr(w_q), _ptr(w_k), _ptr(w_w), _ptr(pos), rows, d_model, h_s, d_s, rope_dim,
        rope_base, _ptr(q_out), _ptr(w_out), _ptr(k_cache), rows_per_seq, l_cap,
        _stream(stream)))


def spot_selector_project_pooled(h, w_q, w_k, w_w, pos, seq_len, n_seq, d_model, h_s, d_s,
                                 rope_dim, rope_base, q_out, w_out, k_cache, k_pool, l_cap,
                                 stream=None):
    if _native is not None:
        st = _native.selector_project_pooled(h, w_q, w_k, w_w, pos, seq_len, n_seq, d_model, h_s,
                                             d_s, rope_dim, rope_base, q_out, w_out, k_cache,
                                             k_pool, l_cap, stream)
        if st is not None:
            return _check("spot_selector_project_pooled", st)
    n_out = h_s * d_s
    _dev(h, "h", BF16, n_seq * d_model)
    _dev(w_q, "w_q", BF16, n_out * d_model)
    _dev(w_k, "w_k", BF16, n_out * d_model)
    _dev(w_w, "w_w", BF16, h_s * d_model)
    _dev(pos, "pos", I32, n_seq)
    if seq_len is not None:
        _dev(seq_len, "seq_len", I32, n_seq)
    _dev(q_out, "q_out", BF16, n_seq * n_out)
    _dev(w_out, "w_out", F32, n_seq * h_s)
    _dev(k_cache, "k_cache", BF16, n_seq * l_cap * n_out)
    _dev(k_pool, "k_pool", BF16, n_seq * (l_cap // BLK) * n_out)
    _check("spot_selector_project_pooled", load().spot_selector_project_pooled(
        _ptr(h), _ptr(w_q), _ptr(w_k), _ptr(w_w), _ptr(pos), _ptr(seq_len), n_seq, d_model, h_s,
        d_s, rope_dim, rope_base, _ptr(q_out), _ptr(w_out), _ptr(k_cache), _ptr(k_pool), l_cap,
        _stream(stream)))


def spot_selector_pool(k_tok, k_pool, n_seq, l_cap, h_s, d_s, seq_len=None, first_block=None,
                       max_blocks=None, stream=None):
    if _native is not None:
        st = _native.selector_pool(k_tok, k_pool, n_seq, l_cap, h_s, d_s, seq_len, first_block,
                                   max_blocks, stream)
        if st is not None:
            return _check("spot_selector_pool", st)
    _dev(k_tok, "k_tok", BF16, n_seq * l_cap * h_s * d_s)
    _dev(k_pool, "k_pool", BF16, n_seq * (l_cap // 64) * h_s * d_s)
    if seq_len is not None:
        _dev(seq_len, "seq_len", I32, n_seq)
    if first_block is not None:
        _dev(first_block, "first_block", I32, n_seq)
    if max_blocks is None:
        max_blocks = l_cap // 64
    _check("spot_selector_pool", load().spot_selector_pool(
        _ptr(k_tok), _ptr(k_pool), n_seq, l_cap, h_s, d_s, _ptr(seq_len), _ptr(first_block),
        max_blocks, _stream(stream)))


def spot_select_blocks(scores, rows, nblk, n_valid, top_p, k_max, k_min, n_sink, n_recent, idx,
                       count, nuc_mass=None, stream=None):
    if _native is not None:
        st = _native.select_blocks(scores, rows, nblk, n_valid, top_p, k_max, k_min, n_sink,
                                   n_recent, idx, count, nuc_mass, stream)
        if st is not None:
            return _check("spot_select_blocks", st)
    _dev(scores, "scores", F32, rows * nblk)
    if n_valid is not None:
        _dev(n_valid, "n_valid", I32, rows)
    _dev(idx, "idx", I32, rows * k_max)
    _dev(count, "count", I32, rows)
    if nuc_mass is not None:
        _dev(nuc_mass, "nuc_mass", F32, rows)
    _check("spot_select_blocks", load().spot_select_blocks(
        _ptr(scores), rows, nblk, _ptr(n_valid), float(top_p), k_max, k_min, n_sink, n_recent,
        _ptr(idx), _ptr(count), _ptr(nuc_mass), _stream(stream)))


def spot_decode_workspace_bytes(batch, h_q, h_kv, d, max_blocks) -> int:
    return int(load().spot_decode_workspace_bytes(batch, h_q, h_kv, d, max_blocks))


def spot_sparse_decode(q, k, v, seq_len, idx, count, k_max, batch, h_q, h_kv, d, l_cap,
                       sm_scale, out, lse, ws, stream=None):
    if _native is not None:
        st = _native.sparse_decode_blk(q, k, v, seq_len, idx, count, k_max, BLK, batch, h_q, h_kv,
                                       d, l_cap, sm_scale, out, lse, ws, stream)
        if st is not None:
            return _check("spot_sparse_decode", st)
    _decode_args(q, k, v, seq_len, idx, count, k_max, batch, h_q, h_kv, d, l_cap, out, lse, ws)
    _check("spot_sparse_decode", load().spot_sparse_decode(
        _ptr(q), _ptr(k), _ptr(v), _ptr(seq_len), _ptr(idx), _ptr(count), k_max, batch, h_q,
        h_kv, d, l_cap, float(sm_scale), _ptr(out), _ptr(lse), _ptr(ws),
        ws.numel() * ws.element_size(), _stream(stream)))


def spot_sparse_decode_blk(q, k, v, seq_len, idx, count, k_max, blk, batch, h_q, h_kv, d, l_cap,
                           sm_scale, out, lse, ws, stream=None):
    if _native is not None:
        st = _native.sparse_decode_blk(q, k, v, seq_len, idx, count, k_max, blk, batch, h_q, h_kv,
                                       d, l_cap, sm_scale, out, lse, ws, stream)
        if st is not None:
            return _check("spot_sparse_decode_blk", st)
    _decode_args(q, k, v, seq_len, idx, count, k_max, batch, h_q, h_kv, d, l_cap, out, lse, ws)
    _check("spot_sparse_decode_blk", load().spot_sparse_decode_blk(
        _ptr(q), _ptr(k), _ptr(v), _ptr(seq_len), _ptr(idx), _ptr(count), k_max, blk, batch,
        h_q, h_kv, d, l_cap, float(sm_scale), _ptr(out), _ptr(lse), _ptr(ws),
        ws.numel() * ws.element_size(), _stream(stream)))


def _decode_args(q, k, v, seq_len, idx, count, k_max, batch, h_q, h_kv, d, l_cap, out, lse, ws):
    _dev(q, "q", BF16, batch * h_q * d)
    _dev(k, "k", BF16, batch * h_kv * l_cap * d)
    _dev(v, "v", BF16, batch * h_kv * l_cap * d)
    _dev(seq_len, "seq_len", I32, batch)
    _dev(idx, "idx", I32, batch * k_max)
    _dev(count, "count", I32, batch)
    _dev(out, "out", BF16, batch * h_q * d)
    if lse is not None:
        _dev(lse, "lse", F32, batch * h_q)
    _dev(ws, "ws", None)


def spot_dense_decode(q, k, v, seq_len, batch, h_q, h_kv, d, l_cap, sm_scale, out, lse, ws,
                      stream=None):
    if _native is not None:
        st = _native.dense_decode(q, k, v, seq_len, batch, h_q, h_kv, d, l_cap, sm_scale, out,
                                  lse, ws, stream)
        if st is not None:
            return _check("spot_dense_decode", st)
    _dev(q, "q", BF16, batch * h_q * d)
    _dev(k, "k", BF16, batch * h_kv * l_cap * d)
    _dev(v, "v", BF16, batch * h_kv * l_cap * d)
    _dev(seq_len, "seq_len", I32, batch)
    _dev(out, "out", BF16, batch * h_q * d)
    if lse is not None:
        _dev(lse, "lse", F32, batch * h_q)
    _dev(ws, "ws", None)
    _check("spot_dense_decode", load().spot_dense_decode(
        _ptr(q), _ptr(k), _ptr(v), _ptr(seq_len), batch, h_q, h_kv, d, l_cap, float(sm_scale),
        _ptr(out), _ptr(lse), _ptr(ws), ws.numel() * ws.element_size(), _stream(stream)))


def spot_sparse_prefill(q, k, v, L, idx, count, k_max, batch, h_q, h_kv, d, sm_scale, out, lse,
                        stream=None):
    if _native is not None:
        st = _native.sparse_prefill(q, k, v, L, idx, count, k_max, batch, h_q, h_kv, d, sm_scale,
                                    out, lse, stream)
        if st is not None:
            return _check("spot_sparse_prefill", st)
    nqb = L // BLK
    _dev(q, "q", BF16, batch * h_q * L * d)
    _dev(k, "k", BF16, batch * h_kv * L * d)
    _dev(v, "v", BF16, batch * h_kv * L * d)
    _dev(idx, "idx", I32, batch * nqb * k_max)
    _dev(count, "count", I32, batch * nqb)
    _dev(out, "out", BF16, batch * h_q * L * d)
    if lse is not None:
        _dev(lse, "lse", F32, batch * h_q * L)
    _check("spot_sparse_prefill", load().spot_sparse_prefill(
        _ptr(q), _ptr(k), _ptr(v), L, _ptr(idx), _ptr(count), k_max, batch, h_q, h_kv, d,
        float(sm_scale), _ptr(out), _ptr(lse), _stream(stream)))


def spot_decode_step_workspace_bytes(batch, h_q, h_kv, d, k_max) -> int:
    return int(load().spot_decode_step_workspace_bytes(batch, h_q, h_kv, d, k_max))


def spot_decode_step(q_sel, w, k_sel, k_scale, kfmt, h_s, d_s, n_valid, top_p, k_max, k_min,
                     n_sink, n_recent, q, k, v, seq_len, batch, h_q, h_kv, d, l_cap, sm_scale,
                     scores, idx, count, nuc_mass, out, lse, ws, stream=None, q_scale=None,
                     qfmt="bf16"):
    """spot_decode_step, or spot_decode_step_q when qfmt is not BF16."""
    if _native is not None:
        st = _native.decode_step(q_sel, w, k_sel, k_scale, kfmt, h_s, d_s, n_valid, top_p, k_max,
                                 k_min, n_sink, n_recent, q, k, v, seq_len, batch, h_q, h_kv, d,
                                 l_cap, sm_scale, scores, idx, count, nuc_mass, out, lse, ws,
                                 stream, q_scale, qfmt)
        if st is not None:
            return _check("spot_decode_step" if qfmt in (0, "bf16") else "spot_decode_step_q",
                          st)
    nblk = l_cap // BLK
    f = KFMT[kfmt] if isinstance(kfmt, str) else int(kfmt)
    qf = KFMT[qfmt] if isinstance(qfmt, str) else int(qfmt)
    _sel_cache(q_sel, q_scale, qf, batch, h_s, d_s, "q_sel", "q_scale")
    _dev(w, "w", F32, batch * h_s)
    _sel_cache(k_sel, k_scale, f, batch * nblk, h_s, d_s, "k_sel")
    if n_valid is not None:
        _dev(n_valid, "n_valid", I32, batch)
    _dev(q, "q", BF16, batch * h_q * d)
    _dev(k, "k", BF16, batch * h_kv * l_cap * d)
    _dev(v, "v", BF16, batch * h_kv * l_cap * d)
    _dev(seq_len, "seq_len", I32, batch)
    _dev(scores, "scores", F32, batch * nblk)
    _dev(idx, "idx", I32, batch * k_max)
    _dev(count, "count", I32, batch)
    if nuc_mass is not None:
        _dev(nuc_mass, "nuc_mass", F32, batch)
    _dev(out, "out", BF16, batch * h_q * d)
    if lse is not None:
        _dev(lse, "lse", F32, batch * h_q)
    _dev(ws, "ws", None)
    rest = (f, h_s, d_s, _ptr(n_valid), float(top_p), k_max, k_min, n_sink, n_recent, _ptr(q),
            _ptr(k), _ptr(v), _ptr(seq_len), batch, h_q, h_kv, d, l_cap, float(sm_scale),
            _ptr(scores), _ptr(idx), _ptr(count), _ptr(nuc_mass), _ptr(out), _ptr(lse), _ptr(ws),
            ws.numel() * ws.element_size(), _stream(stream))
    if qf == 0:
        _check("spot_decode_step", load().spot_decode_step(
            _ptr(q_sel), _ptr(w), _ptr(k_sel), _ptr(k_scale), *rest))
    else:
        _check("spot_decode_step_q", load().spot_decode_step_q(
            _ptr(q_sel), _ptr(q_scale), qf, _ptr(w), _ptr(k_sel), _ptr(k_scale), *rest))


def spot_decode_step_static(q_sel, w, k_sel, k_scale, kfmt, h_s, d_s, n_valid, top_p, k_max,
                            k_min, n_sink, n_recent, q, k, v, seq_len, batch, h_q, h_kv, d, l_cap,
                            sm_scale, scores, idx, count, nuc_mass, out, lse, stream=None):
    """spot_decode_step on the device's static scratch (no workspace argument)."""
    if _native is not None:
        st = _native.decode_step_static(q_sel, w, k_sel, k_scale, kfmt, h_s, d_s, n_valid, top_p,
                                        k_max, k_min, n_sink, n_recent, q, k, v, seq_len, batch,
                                        h_q, h_kv, d, l_cap, sm_scale, scores, idx, count,
                                        nuc_mass, out, lse, stream)
        if st is not None:
            return _check("spot_decode_step_static", st)
    nblk = l_cap // BLK
    f = KFMT[kfmt] if isinstance(kfmt, str) else int(kfmt)
    _dev(q_sel, "q_sel", BF16, batch * h_s * d_s)
    _dev(w, "w", F32, batch * h_s)
    _sel_cache(k_sel, k_scale, f, batch * nblk, h_s, d_s, "k_sel")
    if n_valid is not None:
        _dev(n_valid, "n_valid", I32, batch)
    _dev(q, "q", BF16, batch * h_q * d)
    _dev(k, "k", BF16, batch * h_kv * l_cap * d)
    _dev(v, "v", BF16, batch * h_kv * l_cap * d)
    _dev(seq_len, "seq_len", I32, batch)
    _dev(scores, "scores", F32, batch * nblk)
    _dev(idx, "idx", I32, batch * k_max)
    _dev(count, "count", I32, batch)
    if nuc_mass is not None:
        _dev(nuc_mass, "nuc_mass", F32, batch)
    _dev(out, "out", BF16, batch * h_q * d)
    if lse is not None:
        _dev(lse, "lse", F32, batch * h_q)
    _check("spot_decode_step_static", load().spot_decode_step_static(
        _ptr(q_sel), _ptr(w), _ptr(k_sel), _ptr(k_scale), f, h_s, d_s, _ptr(n_valid),
        float(top_p), k_max, k_min, n_sink, n_recent, _ptr(q), _ptr(k), _ptr(v), _ptr(seq_len),
        batch, h_q, h_kv, d, l_cap, float(sm_scale), _ptr(scores), _ptr(idx), _ptr(count),
        _ptr(nuc_mass), _ptr(out), _ptr(lse), _stream(stream)))


def spot_decode_step_status(ws, batch, h_q, h_kv, d, k_max, stream=None) -> int:
    """Status of a fused-step workspace (ws None: the device's static scratch
    of spot_decode_step_static): SPOT_OK, or SPOT_ERR_EXPIRED after a bounded
    wait expired (the workspace is then zero-filled again).  Any other status
    raises."""
    if ws is not None:
        _dev(ws, "ws", None)
    st = load().spot_decode_step_status(_ptr(ws), 0 if ws is None else ws.numel() * ws.element_size(),
                                        batch, h_q, h_kv, d, k_max, _stream(stream))
    if st not in (SPOT_OK, SPOT_ERR_EXPIRED):
        raise SpotError("spot_decode_step_status", st)
    return int(st)


def spot_test_force_expiry(on: bool):
    load().spot_test_force_expiry(1 if on else 0)


# --------------------------------------------------- operators on a paged cache
def _same_device(stream, *tensors):
    """The device of every tensor given, and its stream: the stream passed, or the
    device's current one."""
    dev = tensors[0].device
    for t in tensors:
        if t is not None and t.device != dev:
            raise ValueError(f"tensors on {dev} and {t.device}")
    if isinstance(stream, torch.cuda.Stream) and stream.device != dev:
        raise ValueError(f"a stream of {stream.device} for tensors on {dev}")
    return dev, _stream(torch.cuda.current_stream(dev) if stream is None else stream)


def _element(t, name):
    """The SPOT_DTYPE of a tensor."""
    if t is None:
        raise ValueError(f"{name} is required")
    if t.dtype not in PAGED_DTYPE:
        raise ValueError(f"{name}: dtype {t.dtype} not in {tuple(PAGED_DTYPE)}")
    return PAGED_DTYPE[t.dtype]


def _opt(t, name, dtypes, numel):
    if t is not None:
        _dev(t, name, dtypes, numel)


def _row_tensor(t, name, dtype, rows, stride, row):
    """Rows of `row` elements, `stride` apart, inside the tensor's storage."""
    if t is None:
        raise ValueError(f"{name} is required")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.dtype != dtype:
        raise ValueError(f"{name}: dtype {t.dtype} is not {dtype}")
    left = t.untyped_storage().nbytes() // t.element_size() - t.storage_offset()
    if rows > 0 and (rows - 1) * stride + row > left:
        raise ValueError(f"{name}: {left} elements, need {(rows - 1) * stride + row}")


def _freq(freq, rope_dim):
    if not isinstance(freq, torch.Tensor) or freq.device.type != "cpu" or \
            freq.dtype != torch.float64 or not freq.is_contiguous():
        raise ValueError("freq must be a contiguous float64 host tensor")
    if freq.numel() < rope_dim // 2:
        raise ValueError(f"freq: {freq.numel()} elements, need {rope_dim // 2}")


def _axis(axis, n_axes, rope_dim):
    """Axes of the pairs; not read where the call has none."""
    if axis is None and n_axes == 0:
        return
    if not isinstance(axis, torch.Tensor) or axis.device.type != "cpu" or \
            axis.dtype != torch.uint8 or not axis.is_contiguous():
        raise ValueError("axis must be a contiguous uint8 host tensor")
    if n_axes > 0 and axis.numel() < rope_dim // 2:
        raise ValueError(f"axis: {axis.numel()} elements, need {rope_dim // 2}")


def _pools8(k_pages, v_pages, k_scale, v_scale, tokens, d):
    """Codes and scales of 8-bit pools of tokens x d elements."""
    _dev(k_pages, "k_pages", CODES8, tokens * d)
    _dev(v_pages, "v_pages", CODES8, tokens * d)
    _dev(k_scale, "k_scale", SCALES8, tokens // 16)
    _dev(v_scale, "v_scale", SCALES8, tokens // 16)


def spot_rope_frequencies(rope_dim, rope_base, scaling, factor, orig_len, low, high, freq):
    _freq(freq, rope_dim)
    _check("spot_rope_frequencies", load().spot_rope_frequencies(
        rope_dim, float(rope_base), scaling, float(factor), orig_len, float(low), float(high),
        _ptr(freq)))


def spot_rotary(x, x_stride, pos, rows, heads, d, rope_dim, freq, amp, flags, out, out_stride,
                stream=None):
    if _native is not None:
        st = _native.rotary(x, x_stride, pos, rows, heads, d, rope_dim, freq, amp, flags, out,
                            out_stride, stream)
        if st is not None:
            return _check("spot_rotary", st)
    dt = _element(x, "x")
    _row_tensor(x, "x", x.dtype, rows, x_stride, heads * d)
    _dev(pos, "pos", I32, rows)
    _freq(freq, rope_dim)
    _row_tensor(out, "out", x.dtype, rows, out_stride, heads * d)
    dev, s = _same_device(stream, x, pos, out)
    with torch.cuda.device(dev):
        _check("spot_rotary", load().spot_rotary(
            _ptr(x), x_stride, _ptr(pos), rows, heads, d, rope_dim, _ptr(freq), float(amp), flags,
            dt, _ptr(out), out_stride, s))


def spot_rotary_append(q, q_stride, k, k_stride, v, v_stride, pos, page_table, n_pages, page_size,
                       max_pages, seq_start, seq_len, n_seq, rows, h_q, h_kv, d, rope_dim, freq,
                       amp, flags, q_out, k_pages, v_pages, stream=None):
    if _native is not None:
        st = _native.rotary_append(q, q_stride, k, k_stride, v, v_stride, pos, page_table, n_pages,
                                   page_size, max_pages, seq_start, seq_len, n_seq, rows, h_q,
                                   h_kv, d, rope_dim, freq, amp, flags, q_out, k_pages, v_pages,
                                   stream)
        if st is not None:
            return _check("spot_rotary_append", st)
    dt = _element(q, "q")
    el = (q.dtype,)
    _row_tensor(q, "q", q.dtype, rows, q_stride, h_q * d)
    _row_tensor(k, "k", q.dtype, rows, k_stride, h_kv * d)
    _row_tensor(v, "v", q.dtype, rows, v_stride, h_kv * d)
    _opt(pos, "pos", I32, rows)
    _dev(page_table, "page_table", I32, n_seq * max_pages)
    _dev(seq_start, "seq_start", I32, n_seq + 1)
    _dev(seq_len, "seq_len", I32, n_seq)
    _freq(freq, rope_dim)
    _dev(q_out, "q_out", el, rows * h_q * d)
    _dev(k_pages, "k_pages", el, n_pages * h_kv * page_size * d)
    _dev(v_pages, "v_pages", el, n_pages * h_kv * page_size * d)
    dev, s = _same_device(stream, q, k, v, pos, page_table, seq_start, seq_len, q_out, k_pages,
                          v_pages)
    with torch.cuda.device(dev):
        _check("spot_rotary_append", load().spot_rotary_append(
            _ptr(q), q_stride, _ptr(k), k_stride, _ptr(v), v_stride, dt, _ptr(pos),
            _ptr(page_table), n_pages, page_size, max_pages, _ptr(seq_start), _ptr(seq_len),
            n_seq, rows, h_q, h_kv, d, rope_dim, _ptr(freq), float(amp), flags, _ptr(q_out),
            _ptr(k_pages), _ptr(v_pages), s))


def spot_paged_workspace_bytes(n_seq, rows, h_q, h_kv, d) -> int:
    return int(load().spot_paged_workspace_bytes(n_seq, rows, h_q, h_kv, d))


def spot_paged_attend(q, k_pages, v_pages, page_table, n_pages, page_size, max_pages, seq_start,
                      seq_len, n_seq, rows, h_q, h_kv, d, sm_scale, softcap, slopes, window,
                      prefix, first, out, lse, ws, stream=None):
    if _native is not None:
        st = _native.paged_attend(q, k_pages, v_pages, page_table, n_pages, page_size, max_pages,
                                  seq_start, seq_len, n_seq, rows, h_q, h_kv, d, sm_scale, softcap,
                                  slopes, window, prefix, first, out, lse, ws, stream)
        if st is not None:
            return _check("spot_paged_attend", st)
    dt = _element(q, "q")
    el = (q.dtype,)
    _dev(q, "q", el, rows * h_q * d)
    _dev(k_pages, "k_pages", el, n_pages * h_kv * page_size * d)
    _dev(v_pages, "v_pages", el, n_pages * h_kv * page_size * d)
    _dev(page_table, "page_table", I32, n_seq * max_pages)
    _dev(seq_start, "seq_start", I32, n_seq + 1)
    _dev(seq_len, "seq_len", I32, n_seq)
    _opt(slopes, "slopes", F32, h_q)
    _opt(prefix, "prefix", I32, n_seq)
    _opt(first, "first", I32, rows)
    _dev(out, "out", el, rows * h_q * d)
    _opt(lse, "lse", F32, rows * h_q)
    _dev(ws, "ws", None)
    dev, s = _same_device(stream, q, k_pages, v_pages, page_table, seq_start, seq_len, slopes,
                          prefix, first, out, lse, ws)
    with torch.cuda.device(dev):
        _check("spot_paged_attend", load().spot_paged_attend(
            _ptr(q), dt, _ptr(k_pages), _ptr(v_pages), _ptr(page_table), n_pages, page_size,
            max_pages, _ptr(seq_start), _ptr(seq_len), n_seq, rows, h_q, h_kv, d, float(sm_scale),
            float(softcap), _ptr(slopes), window, _ptr(prefix), _ptr(first), _ptr(out), _ptr(lse),
            _ptr(ws), ws.numel() * ws.element_size(), s))


def spot_paged_weights(q, lse, k_pages, page_table, n_pages, page_size, max_pages, seq_start,
                       seq_len, n_seq, rows, h_q, h_kv, d, sm_scale, softcap, slopes, window,
                       prefix, first, acc, decay, acc_out, stream=None):
    if _native is not None:
        st = _native.paged_weights(q, lse, k_pages, page_table, n_pages, page_size, max_pages,
                                   seq_start, seq_len, n_seq, rows, h_q, h_kv, d, sm_scale,
                                   softcap, slopes, window, prefix, first, acc, decay, acc_out,
                                   stream)
        if st is not None:
            return _check("spot_paged_weights", st)
    dt = _element(q, "q")
    el = (q.dtype,)
    _dev(q, "q", el, rows * h_q * d)
    _dev(lse, "lse", F32, rows * h_q)
    _dev(k_pages, "k_pages", el, n_pages * h_kv * page_size * d)
    _dev(page_table, "page_table", I32, n_seq * max_pages)
    _dev(seq_start, "seq_start", I32, n_seq + 1)
    _dev(seq_len, "seq_len", I32, n_seq)
    _opt(slopes, "slopes", F32, h_q)
    _opt(prefix, "prefix", I32, n_seq)
    _opt(first, "first", I32, rows)
    _opt(acc, "acc", F32, n_seq * h_kv * max_pages * page_size)
    _dev(acc_out, "acc_out", F32, n_seq * h_kv * max_pages * page_size)
    dev, s = _same_device(stream, q, lse, k_pages, page_table, seq_start, seq_len, slopes, prefix,
                          first, acc, acc_out)
    with torch.cuda.device(dev):
        _check("spot_paged_weights", load().spot_paged_weights(
            _ptr(q), _ptr(lse), dt, _ptr(k_pages), _ptr(page_table), n_pages, page_size, max_pages,
            _ptr(seq_start), _ptr(seq_len), n_seq, rows, h_q, h_kv, d, float(sm_scale),
            float(softcap), _ptr(slopes), window, _ptr(prefix), _ptr(first), _ptr(acc),
            float(decay), _ptr(acc_out), s))


def spot_cache_evict(acc, k_pages, v_pages, page_table, n_pages, page_size, max_pages, seq_len,
                     n_seq, h_kv, d, budget, n_sink, n_recent, k_dst, v_dst, dst_table,
                     n_dst_pages, dst_max_pages, idx, new_len, acc_out, out_cap, stream=None):
    if _native is not None:
        st = _native.cache_evict(acc, k_pages, v_pages, page_table, n_pages, page_size, max_pages,
                                 seq_len, n_seq, h_kv, d, budget, n_sink, n_recent, k_dst, v_dst,
                                 dst_table, n_dst_pages, dst_max_pages, idx, new_len, acc_out,
                                 out_cap, stream)
        if st is not None:
            return _check("spot_cache_evict", st)
    _element(k_pages, "k_pages")
    el = (k_pages.dtype,)
    page = h_kv * page_size * d
    _dev(acc, "acc", F32, n_seq * h_kv * max_pages * page_size)
    _dev(k_pages, "k_pages", el, n_pages * page)
    _dev(v_pages, "v_pages", el, n_pages * page)
    _dev(page_table, "page_table", I32, n_seq * max_pages)
    _dev(seq_len, "seq_len", I32, n_seq)
    _dev(k_dst, "k_dst", el, n_dst_pages * page)
    _dev(v_dst, "v_dst", el, n_dst_pages * page)
    _dev(dst_table, "dst_table", I32, n_seq * dst_max_pages)
    _dev(idx, "idx", I32, n_seq * h_kv * budget)
    _dev(new_len, "new_len", I32, n_seq)
    _dev(acc_out, "acc_out", F32, n_seq * h_kv * out_cap)
    dev, s = _same_device(stream, acc, k_pages, v_pages, page_table, seq_len, k_dst, v_dst,
                          dst_table, idx, new_len, acc_out)
    with torch.cuda.device(dev):
        _check("spot_cache_evict", load().spot_cache_evict(
            _ptr(acc), _ptr(k_pages), _ptr(v_pages), _ptr(page_table), n_pages, page_size,
            max_pages, _ptr(seq_len), n_seq, h_kv, d, budget, n_sink, n_recent, _ptr(k_dst),
            _ptr(v_dst), _ptr(dst_table), n_dst_pages, dst_max_pages, _ptr(idx), _ptr(new_len),
            _ptr(acc_out), out_cap, s))


def spot_rotary_axes(x, x_stride, pos, n_axes, axis, rows, heads, d, rope_dim, freq, amp, flags,
                     out, out_stride, stream=None):
    if _native is not None:
        st = _native.rotary_axes(x, x_stride, pos, n_axes, axis, rows, heads, d, rope_dim, freq,
                                 amp, flags, out, out_stride, stream)
        if st is not None:
            return _check("spot_rotary_axes", st)
    dt = _element(x, "x")
    _row_tensor(x, "x", x.dtype, rows, x_stride, heads * d)
    _dev(pos, "pos", I32, rows * max(n_axes, 1))
    _axis(axis, n_axes, rope_dim)
    _freq(freq, rope_dim)
    _row_tensor(out, "out", x.dtype, rows, out_stride, heads * d)
    dev, s = _same_device(stream, x, pos, out)
    with torch.cuda.device(dev):
        _check("spot_rotary_axes", load().spot_rotary_axes(
            _ptr(x), x_stride, _ptr(pos), n_axes, _ptr(axis), rows, heads, d, rope_dim, _ptr(freq),
            float(amp), flags, dt, _ptr(out), out_stride, s))


def spot_rotary_append8(q, q_stride, k, k_stride, v, v_stride, pos, n_axes, axis, page_table,
                        n_pages, page_size, max_pages, seq_start, seq_len, n_seq, rows, h_q, h_kv,
                        d, rope_dim, freq, amp, flags, q_out, k_pages, v_pages, k_scale, v_scale,
                        stream=None):
    if _native is not None:
        st = _native.rotary_append8(q, q_stride, k, k_stride, v, v_stride, pos, n_axes, axis,
                                    page_table, n_pages, page_size, max_pages, seq_start, seq_len,
                                    n_seq, rows, h_q, h_kv, d, rope_dim, freq, amp, flags, q_out,
                                    k_pages, v_pages, k_scale, v_scale, stream)
        if st is not None:
            return _check("spot_rotary_append8", st)
    dt = _element(q, "q")
    el = (q.dtype,)
    _row_tensor(q, "q", q.dtype, rows, q_stride, h_q * d)
    _row_tensor(k, "k", q.dtype, rows, k_stride, h_kv * d)
    _row_tensor(v, "v", q.dtype, rows, v_stride, h_kv * d)
    _opt(pos, "pos", I32, rows * max(n_axes, 1))
    _axis(axis, n_axes, rope_dim)
    _dev(page_table, "page_table", I32, n_seq * max_pages)
    _dev(seq_start, "seq_start", I32, n_seq + 1)
    _dev(seq_len, "seq_len", I32, n_seq)
    _freq(freq, rope_dim)
    _dev(q_out, "q_out", el, rows * h_q * d)
    _pools8(k_pages, v_pages, k_scale, v_scale, n_pages * h_kv * page_size, d)
    dev, s = _same_device(stream, q, k, v, pos, page_table, seq_start, seq_len, q_out, k_pages,
                          v_pages, k_scale, v_scale)
    with torch.cuda.device(dev):
        _check("spot_rotary_append8", load().spot_rotary_append8(
            _ptr(q), q_stride, _ptr(k), k_stride, _ptr(v), v_stride, dt, _ptr(pos),
            n_axes, _ptr(axis), _ptr(page_table), n_pages, page_size, max_pages, _ptr(seq_start),
            _ptr(seq_len), n_seq, rows, h_q, h_kv, d, rope_dim, _ptr(freq), float(amp), flags,
            _ptr(q_out), _ptr(k_pages), _ptr(v_pages), _ptr(k_scale), _ptr(v_scale), s))


def spot_paged_attend_sinks(q, k_pages, v_pages, page_table, n_pages, page_size, max_pages,
                            seq_start, seq_len, n_seq, rows, h_q, h_kv, d, sm_scale, softcap,
                            slopes, window, n_sink, prefix, first, out, lse, ws, stream=None):
    if _native is not None:
        st = _native.paged_attend_sinks(q, k_pages, v_pages, page_table, n_pages, page_size,
                                        max_pages, seq_start, seq_len, n_seq, rows, h_q, h_kv, d,
                                        sm_scale, softcap, slopes, window, n_sink, prefix, first,
                                        out, lse, ws, stream)
        if st is not None:
            return _check("spot_paged_attend_sinks", st)
    dt = _element(q, "q")
    el = (q.dtype,)
    _dev(q, "q", el, rows * h_q * d)
    _dev(k_pages, "k_pages", el, n_pages * h_kv * page_size * d)
    _dev(v_pages, "v_pages", el, n_pages * h_kv * page_size * d)
    _dev(page_table, "page_table", I32, n_seq * max_pages)
    _dev(seq_start, "seq_start", I32, n_seq + 1)
    _dev(seq_len, "seq_len", I32, n_seq)
    _opt(slopes, "slopes", F32, h_q)
    _opt(prefix, "prefix", I32, n_seq)
    _opt(first, "first", I32, rows)
    _dev(out, "out", el, rows * h_q * d)
    _opt(lse, "lse", F32, rows * h_q)
    _dev(ws, "ws", None)
    dev, s = _same_device(stream, q, k_pages, v_pages, page_table, seq_start, seq_len, slopes,
                          prefix, first, out, lse, ws)
    with torch.cuda.device(dev):
        _check("spot_paged_attend_sinks", load().spot_paged_attend_sinks(
            _ptr(q), dt, _ptr(k_pages), _ptr(v_pages), _ptr(page_table), n_pages, page_size,
            max_pages, _ptr(seq_start), _ptr(seq_len), n_seq, rows, h_q, h_kv, d, float(sm_scale),
            float(softcap), _ptr(slopes), window, n_sink, _ptr(prefix), _ptr(first), _ptr(out),
            _ptr(lse), _ptr(ws), ws.numel() * ws.element_size(), s))


def spot_paged_attend8(q, k_pages, v_pages, k_scale, v_scale, page_table, n_pages, page_size,
                       max_pages, seq_start, seq_len, n_seq, rows, h_q, h_kv, d, sm_scale, softcap,
                       slopes, window, n_sink, prefix, first, out, lse, ws, stream=None):
    if _native is not None:
        st = _native.paged_attend8(q, k_pages, v_pages, k_scale, v_scale, page_table, n_pages,
                                   page_size, max_pages, seq_start, seq_len, n_seq, rows, h_q, h_kv,
                                   d, sm_scale, softcap, slopes, window, n_sink, prefix, first, out,
                                   lse, ws, stream)
        if st is not None:
            return _check("spot_paged_attend8", st)
    dt = _element(q, "q")
    el = (q.dtype,)
    _dev(q, "q", el, rows * h_q * d)
    _pools8(k_pages, v_pages, k_scale, v_scale, n_pages * h_kv * page_size, d)
    _dev(page_table, "page_table", I32, n_seq * max_pages)
    _dev(seq_start, "seq_start", I32, n_seq + 1)
    _dev(seq_len, "seq_len", I32, n_seq)
    _opt(slopes, "slopes", F32, h_q)
    _opt(prefix, "prefix", I32, n_seq)
    _opt(first, "first", I32, rows)
    _dev(out, "out", el, rows * h_q * d)
    _opt(lse, "lse", F32, rows * h_q)
    _dev(ws, "ws", None)
    dev, s = _same_device(stream, q, k_pages, v_pages, k_scale, v_scale, page_table, seq_start,
                          seq_len, slopes, prefix, first, out, lse, ws)
    with torch.cuda.device(dev):
        _check("spot_paged_attend8", load().spot_paged_attend8(
            _ptr(q), dt, _ptr(k_pages), _ptr(v_pages), _ptr(k_scale), _ptr(v_scale),
            _ptr(page_table), n_pages, page_size, max_pages, _ptr(seq_start), _ptr(seq_len), n_seq,
            rows, h_q, h_kv, d, float(sm_scale), float(softcap), _ptr(slopes), window, n_sink,
            _ptr(prefix), _ptr(first), _ptr(out), _ptr(lse), _ptr(ws),
            ws.numel() * ws.element_size(), s))


def spot_probe_stream_read(buf, sink, stream=None):
    _dev(buf, "buf", None)
    _dev(sink, "sink", F32, int(load().spot_probe_sink_words()))
    _check("spot_probe_stream_read", load().spot_probe_stream_read(
        _ptr(buf), buf.numel() * buf.element_size(), _ptr(sink), _stream(stream)))


# --------------------------------------------------- allocating wrappers
_HERE = contextlib.nullcontext()


def _on(stream, device):
    """The context in which a wrapper makes what the caller left out: the call's stream.
    What fills a tensor has to come before the kernel, and its memory may not be given to
    another stream's work while the kernel runs."""
    if stream is None or device.type == "cpu":
        return _HERE
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(int(stream), device) if int(stream) else \
            torch.cuda.default_stream(device)
    return torch.cuda.stream(stream)


def selector_score(q_sel, w, k_sel, k_scale=None, kfmt="bf16", rows_per_seq=1, n_valid=None,
                   nblk=None, out=None, stream=None):
    """Block scores [rows, nblk] float32 for q_sel [rows, h_s, d_s]."""
    h_s, d_s = q_sel.shape[-2], q_sel.shape[-1]
    rows = q_sel.numel() // (h_s * d_s)
    n_seq = rows // rows_per_seq
    if nblk is None:
        f = KFMT.get(kfmt, kfmt)
        per = h_s * d_s if f in (0, 3, 4) else h_s * d_s // 2
        nblk = k_sel.numel() // (n_seq * per)
    if out is None:
        with _on(stream, q_sel.device):
            out = torch.empty((rows, nblk), dtype=torch.float32, device=q_sel.device)
    spot_selector_score(q_sel, w, k_sel, k_scale, kfmt, n_seq, rows_per_seq, nblk, h_s, d_s,
                        n_valid, out, stream)
    return out


def selector_score_tokens(q_sel, w, k_tok, k_scale=None, kfmt="bf16", rows_per_seq=1,
                          seq_len=None, l_cap=None, out=None, stream=None, blk=64):
    """Per-block maximum of per-token scores [rows, l_cap // blk] float32
    (blocks of 64 tokens, or 16: the paper's selector block)."""
    h_s, d_s = q_sel.shape[-2], q_sel.shape[-1]
    rows = q_sel.numel() // (h_s * d_s)
    n_seq = rows // rows_per_seq
    if l_cap is None:
        f = KFMT.get(kfmt, kfmt)
        per = h_s * d_s if f in (0, 3, 4) else h_s * d_s // 2
        l_cap = k_tok.numel() // (n_seq * per)
    if out is None:
        with _on(stream, q_sel.device):
            out = torch.empty((rows, l_cap // blk), dtype=torch.float32, device=q_sel.device)
    if blk == 64:
        spot_selector_score_tokens(q_sel, w, k_tok, k_scale, kfmt, n_seq, rows_per_seq, l_cap,
                                   h_s, d_s, seq_len, out, stream)
    else:
        spot_selector_score_tokens_blk(q_sel, w, k_tok, k_scale, kfmt, n_seq, rows_per_seq,
                                       l_cap, blk, h_s, d_s, seq_len, out, stream)
    return out


def select_blocks(scores, rule, n_valid=None, idx=None, count=None, nuc_mass=None, stream=None):
    rows, nblk = scores.shape
    dev = scores.device
    if idx is None or count is None or nuc_mass is None:
        with _on(stream, dev):
            if idx is None:
                idx = torch.empty((rows, rule.k_max), dtype=torch.int32, device=dev)
            if count is None:
                count = torch.empty(rows, dtype=torch.int32, device=dev)
            if nuc_mass is None:
                nuc_mass = torch.empty(rows, dtype=torch.float32, device=dev)
    spot_select_blocks(scores, rows, nblk, n_valid, rule.top_p, rule.k_max, rule.k_min,
                       rule.n_sink, rule.n_recent, idx, count, nuc_mass, stream)
    return idx, count, nuc_mass


def decode_workspace(batch, h_q, h_kv, d, max_blocks, device="cuda"):
    """Zero-filled decode workspace (the library keeps it zeroed between calls)."""
    n = spot_decode_workspace_bytes(batch, h_q, h_kv, d, max_blocks)
    return torch.zeros(max(n, 16), dtype=torch.uint8, device=device)


def sparse_decode(q, k, v, seq_len, idx, count, sm_scale=None, out=None, lse=None, ws=None,
                  stream=None, blk=64):
    """Attention over the selected blocks of blk tokens (64, or 16: the
    paper's selector block); returns (out [batch, h_q, d] BF16, lse)."""
    batch, h_q, d = q.shape
    _, h_kv, l_cap, _ = k.shape
    k_max = idx.shape[-1]
    sm_scale = 1.0 / math.sqrt(d) if sm_scale is None else sm_scale
    if out is None or lse is None or ws is None:
        with _on(stream, q.device):
            if out is None:
                out = torch.empty((batch, h_q, d), dtype=torch.bfloat16, device=q.device)
            if lse is None:
                lse = torch.empty((batch, h_q), dtype=torch.float32, device=q.device)
            if ws is None:
                ws = decode_workspace(batch, h_q, h_kv, d, k_max, q.device)
    if blk == 64:
        spot_sparse_decode(q, k, v, seq_len, idx, count, k_max, batch, h_q, h_kv, d, l_cap,
                           sm_scale, out, lse, ws, stream)
    else:
        spot_sparse_decode_blk(q, k, v, seq_len, idx, count, k_max, blk, batch, h_q, h_kv, d,
                               l_cap, sm_scale, out, lse, ws, stream)
    return out, lse


def dense_decode(q, k, v, seq_len, sm_scale=None, out=None, lse=None, ws=None, stream=None):
    batch, h_q, d = q.shape
    _, h_kv, l_cap, _ = k.shape
    sm_scale = 1.0 / math.sqrt(d) if sm_scale is None else sm_scale
    if out is None or lse is None or ws is None:
        with _on(stream, q.device):
            if out is None:
                out = torch.empty((batch, h_q, d), dtype=torch.bfloat16, device=q.device)
            if lse is None:
                lse = torch.empty((batch, h_q), dtype=torch.float32, device=q.device)
            if ws is None:
                ws = decode_workspace(batch, h_q, h_kv, d, l_cap // BLK, q.device)
    spot_dense_decode(q, k, v, seq_len, batch, h_q, h_kv, d, l_cap, sm_scale, out, lse, ws,
                      stream)
    return out, lse


def sparse_prefill(q, k, v, idx, count, sm_scale=None, out=None, lse=None, stream=None):
    batch, h_q, L, d = q.shape
    h_kv = k.shape[1]
    k_max = idx.shape[-1]
    sm_scale = 1.0 / math.sqrt(d) if sm_scale is None else sm_scale
    if out is None or lse is None:
        with _on(stream, q.device):
            if out is None:
                out = torch.empty_like(q, dtype=torch.bfloat16)
            if lse is None:
                lse = torch.empty((batch, h_q, L), dtype=torch.float32, device=q.device)
    spot_sparse_prefill(q, k, v, L, idx, count, k_max, batch, h_q, h_kv, d, sm_scale, out, lse,
                        stream)
    return out, lse


def step_workspace(batch, h_q, h_kv, d, k_max, device="cuda"):
    """Zero-filled workspace of spot_decode_step (kept zeroed between calls)."""
    n = spot_decode_step_workspace_bytes(batch, h_q, h_kv, d, k_max)
    return torch.zeros(max(n, 16), dtype=torch.uint8, device=device)


def decode_step(q_sel, w, k_sel, q, k, v, seq_len, rule, k_scale=None, kfmt="bf16",
                n_valid=None, sm_scale=None, ws=None, stream=None, q_scale=None, qfmt="bf16"):
    """One fused decode step: (scores, idx, count, nuc_mass, out, lse).
    Quantized queries (qfmt = kfmt, codes in q_sel) go through spot_decode_step_q."""
    batch, h_q, d = q.shape
    _, h_kv, l_cap, _ = k.shape
    qf = KFMT[qfmt] if isinstance(qfmt, str) else int(qfmt)
    h_s, d_s = q_sel.shape[-2], q_sel.shape[-1] * (2 if qf in (1, 2) else 1)   # 4-bit codes
    nblk = l_cap // BLK
    dev = q.device
    sm_scale = 1.0 / math.sqrt(d) if sm_scale is None else sm_scale
    with _on(stream, dev):
        scores = torch.empty((batch, nblk), dtype=torch.float32, device=dev)
        idx = torch.empty((batch, rule.k_max), dtype=torch.int32, device=dev)
        count = torch.empty(batch, dtype=torch.int32, device=dev)
        mass = torch.empty(batch, dtype=torch.float32, device=dev)
        out = torch.empty((batch, h_q, d), dtype=torch.bfloat16, device=dev)
        lse = torch.empty((batch, h_q), dtype=torch.float32, device=dev)
        if ws is None:
            ws = step_workspace(batch, h_q, h_kv, d, rule.k_max, dev)
    spot_decode_step(q_sel, w, k_sel, k_scale, kfmt, h_s, d_s, n_valid, rule.top_p, rule.k_max,
                     rule.k_min, rule.n_sink, rule.n_recent, q, k, v, seq_len, batch, h_q, h_kv,
                     d, l_cap, sm_scale, scores, idx, count, mass, out, lse, ws, stream,
                     q_scale=q_scale, qfmt=qfmt)
    return scores, idx, count, mass, out, lse


# ----------------------------------------------- paged cache, allocating wrappers
def rope_frequencies(rope_dim, base=1.0e6, scaling="none", factor=1.0, orig_len=0, low=1.0,
                     high=32.0):
    """Rotary frequencies (float64 host tensor [rope_dim / 2], kept by the caller) and
    the factor on sine and cosine.  scaling: "none", "linear", "ntk" (the base grows),
    "parts" (by the turns of a pair over orig_len tokens, low and high), "yarn" (by
    parts, with YaRN's factor 0.1 ln(factor) + 1)."""
    if scaling not in ROPE_SCALING:
        raise ValueError(f"scaling {scaling!r} not in {tuple(ROPE_SCALING)}")
    freq = torch.empty(max(int(rope_dim), 0) // 2, dtype=torch.float64)
    spot_rope_frequencies(rope_dim, base, ROPE_SCALING[scaling], factor, orig_len, low, high, freq)
    return freq, 0.1 * math.log(factor) + 1.0 if scaling == "yarn" else 1.0


def _shape(t, name, n, *rest):
    """[n or more, *rest]"""
    if t is not None and (tuple(t.shape[1:]) != rest or t.shape[0] < n):
        raise ValueError(f"{name}: shape {tuple(t.shape)}, need {(n, *rest)}")


def _fits(q, k, v, out, cap, acc, acc_out, *pools):
    """The shapes that belong together: pools [*, h_kv, page_size, d] alike, the values' with the
    pages of the keys' before them or more, q [rows, *, d], k and v [rows or more, h_kv, d], out
    [rows or more, heads of q, d], rows of acc and acc_out of cap weights."""
    if _native is not None and _native.paged_fits(q, k, v, out, cap, acc, acc_out, *pools):
        return
    h_kv = page = d = n = None
    for i, (name, p) in enumerate(zip(("k_pages", "v_pages", "k_dst", "v_dst"), pools)):
        if h_kv is None:
            _, h_kv, page, d = p.shape
        if q is not None:
            d = q.shape[2]
        _shape(p, name, n if i % 2 else 0, h_kv, page, d)
        n = p.shape[0]
    if q is not None:
        rows, heads, d = q.shape
        _shape(k, "k", rows, h_kv, d)
        _shape(v, "v", rows, h_kv, d)
        _shape(out, "out", rows, heads, d)
    for name, t in (("acc", acc), ("acc_out", acc_out)):
        if t is not None and t.shape[-1] != cap:
            raise ValueError(f"{name}: rows of {t.shape[-1]} weights for {cap} tokens")


def _strides(t, name):
    """Row stride of [rows, heads, d] whose heads lie one after the other."""
    rows, heads, d = t.shape
    row, head, one = t.stride()
    if (d > 1 and one != 1) or (heads > 1 and head != d):
        raise ValueError(f"{name}: the heads of a row must lie one after the other")
    return row if rows > 1 else heads * d


def _axes_of(axis, pos, freq, rows):
    """The number of axes of positions [rows, axes] with the axis of each pair.  Without an axis
    there is one number a row, in any shape but that."""
    if axis is None:
        if pos is not None and pos.dim() > 1 and 0 < rows <= pos.shape[0] < pos.numel():
            raise ValueError(f"pos: shape {tuple(pos.shape)} for {rows} rows needs the axis of "
                             "every frequency")
        return 0
    if pos is None or pos.dim() != 2 or axis.numel() != freq.numel():
        raise ValueError("axis: need pos [rows, axes] and an axis for every frequency")
    return pos.shape[1]


def rotary(x, pos, freq, amp=1.0, interleaved=False, inverse=False, out=None, stream=None,
           axis=None):
    """Rotary positions of x [rows, heads, d] (rows may be strided): the first
    2 len(freq) elements of each head, pairs (i, i + len(freq)) or neighbours.
    inverse: by the negative angles (also the gradient of the rotation).
    axis (uint8 host tensor, one for every frequency): pair i turns by pos[row, axis[i]] of
    pos [rows, axes], which without it is refused."""
    flags = (ROPE_INTERLEAVED if interleaved else 0) | (ROPE_INVERSE if inverse else 0)
    if axis is not None and out is not None and _native is not None:
        st = _native.rotary_axes_of(x, pos, freq, amp, flags, out, stream, axis)
        if st is not None:
            _check("spot_rotary_axes", st)
            return out
    rows, heads, d = x.shape
    if out is None:
        with _on(stream, x.device):
            out = torch.empty((rows, heads, d), dtype=x.dtype, device=x.device)
    else:
        _fits(x, None, None, out, 0, None, None)
    n_axes = _axes_of(axis, pos, freq, rows)
    if n_axes:
        spot_rotary_axes(x, _strides(x, "x"), pos, n_axes, axis, rows, heads, d, 2 * freq.numel(),
                         freq, amp, flags, out, _strides(out, "out"), stream)
    else:
        spot_rotary(x, _strides(x, "x"), pos, rows, heads, d, 2 * freq.numel(), freq, amp, flags,
                    out, _strides(out, "out"), stream)
    return out


def rotary_append(q, k, v, k_pages, v_pages, page_table, seq_start, seq_len, freq, amp=1.0,
                  interleaved=False, pos=None, q_out=None, stream=None):
    """Rotates q [rows, h_q, d] into q_out and k [rows, h_kv, d] into the pages of a
    paged cache (see spot_paged_attend), and stores v beside it; returns q_out."""
    rows, h_q, d = q.shape
    n_pages, h_kv, page, _ = k_pages.shape
    _fits(q, k, v, q_out, 0, None, None, k_pages, v_pages)
    _axes_of(None, pos, freq, rows)
    if q_out is None:
        with _on(stream, q.device):
            q_out = torch.empty((rows, h_q, d), dtype=q.dtype, device=q.device)
    spot_rotary_append(q, _strides(q, "q"), k, _strides(k, "k"), v, _strides(v, "v"), pos,
                       page_table, n_pages, page, page_table.shape[1], seq_start, seq_len,
                       seq_len.shape[0], rows, h_q, h_kv, d, 2 * freq.numel(), freq, amp,
                       ROPE_INTERLEAVED if interleaved else 0, q_out, k_pages, v_pages, stream)
    return q_out


def _scales(k_scale, v_scale, n_pages, h_kv, page):
    """The scales of 8-bit pools: [n_pages or more, h_kv, page_size / 16]."""
    _shape(k_scale, "k_scale", n_pages, h_kv, page // 16)
    _shape(v_scale, "v_scale", n_pages, h_kv, page // 16)


def rotary_append8(q, k, v, k_pages, v_pages, k_scale, v_scale, page_table, seq_start, seq_len,
                   freq, amp=1.0, interleaved=False, pos=None, q_out=None, stream=None, axis=None):
    """rotary_append into an 8-bit paged cache: e4m3 codes k_pages, v_pages [n_pages, h_kv,
    page_size, d] (uint8 or float8_e4m3fn) and a power of two for every 16 tokens of a head,
    k_scale, v_scale [n_pages, h_kv, page_size / 16] (uint8 or float8_e8m0fnu).  axis and pos
    [rows, axes] as in rotary.  Returns q_out."""
    flags = ROPE_INTERLEAVED if interleaved else 0
    if q_out is not None and _native is not None:
        st = _native.rotary_append8_of(q, k, v, k_pages, v_pages, k_scale, v_scale, page_table,
                                       seq_start, seq_len, freq, amp, flags, pos, q_out, stream,
                                       axis)
        if st is not None:
            _check("spot_rotary_append8", st)
            return q_out
    rows, h_q, d = q.shape
    n_pages, h_kv, page, _ = k_pages.shape
    _fits(q, k, v, q_out, 0, None, None, k_pages, v_pages)
    _scales(k_scale, v_scale, n_pages, h_kv, page)
    if q_out is None:
        with _on(stream, q.device):
            q_out = torch.empty((rows, h_q, d), dtype=q.dtype, device=q.device)
    spot_rotary_append8(q, _strides(q, "q"), k, _strides(k, "k"), v, _strides(v, "v"), pos,
                        _axes_of(axis, pos, freq, rows), axis, page_table, n_pages, page,
                        page_table.shape[1], seq_start, seq_len, seq_len.shape[0], rows, h_q, h_kv,
                        d, 2 * freq.numel(), freq, amp, flags, q_out, k_pages, v_pages, k_scale,
                        v_scale, stream)
    return q_out


def paged_workspace(n_seq, rows, h_q, h_kv, d, device="cuda"):
    """Workspace of paged_attend for calls of at most n_seq sequences and rows rows, its
    counters at zero (each call leaves it ready for the next)."""
    n = spot_paged_workspace_bytes(n_seq, rows, h_q, h_kv, d)
    ws = torch.empty(max(n, 16), dtype=torch.uint8, device=device)
    ws[:PAGED_WORKSPACE_ZEROS].zero_()
    return ws


def _attend_outputs(q, out, lse, ws, n_seq, h_kv, stream):
    """What an attention's caller left out, made on the call's stream."""
    rows, h_q, d = q.shape
    with _on(stream, q.device):
        if out is None:
            out = torch.zeros((rows, h_q, d), dtype=q.dtype, device=q.device)
        if lse is None:
            lse = torch.full((rows, h_q), -math.inf, dtype=torch.float32, device=q.device)
        if ws is None:
            ws = paged_workspace(n_seq, rows, h_q, h_kv, d, q.device)
    return out, lse, ws


def paged_attend(q, k_pages, v_pages, page_table, seq_start, seq_len, sm_scale=None, softcap=0.0,
                 slopes=None, window=0, prefix=None, first=None, out=None, lse=None, ws=None,
                 stream=None, n_sink=0):
    """Attention of the packed new tokens q [rows, h_q, d] of every sequence over its
    pages; k_pages, v_pages [n_pages, h_kv, page_size, d], page_table [n_seq,
    max_pages].  n_sink: as many first tokens (of the sequence, or from first on) stay visible
    before the window.  Returns (out [rows, h_q, d], lse [rows, h_q])."""
    rows, h_q, d = q.shape
    n_pages, h_kv, page, _ = k_pages.shape
    _fits(q, None, None, out, 0, None, None, k_pages, v_pages)
    n_seq, max_pages = page_table.shape
    if sm_scale is None:
        sm_scale = 1.0 / math.sqrt(d)
    if out is None or lse is None or ws is None:
        out, lse, ws = _attend_outputs(q, out, lse, ws, n_seq, h_kv, stream)
    if n_sink:
        spot_paged_attend_sinks(q, k_pages, v_pages, page_table, n_pages, page, max_pages,
                                seq_start, seq_len, n_seq, rows, h_q, h_kv, d, sm_scale, softcap,
                                slopes, window, n_sink, prefix, first, out, lse, ws, stream)
        return out, lse
    spot_paged_attend(q, k_pages, v_pages, page_table, n_pages, page, max_pages, seq_start,
                      seq_len, n_seq, rows, h_q, h_kv, d, sm_scale, softcap, slopes, window,
                      prefix, first, out, lse, ws, stream)
    return out, lse


def paged_attend8(q, k_pages, v_pages, k_scale, v_scale, page_table, seq_start, seq_len,
                  sm_scale=None, softcap=0.0, slopes=None, window=0, n_sink=0, prefix=None,
                  first=None, out=None, lse=None, ws=None, stream=None):
    """paged_attend over an 8-bit cache (see rotary_append8): the elements are
    code * 2^(scale - 127).  Returns (out [rows, h_q, d] of q's type, lse [rows, h_q])."""
    rows, h_q, d = q.shape
    n_pages, h_kv, page, _ = k_pages.shape
    _fits(q, None, None, out, 0, None, None, k_pages, v_pages)
    _scales(k_scale, v_scale, n_pages, h_kv, page)
    n_seq, max_pages = page_table.shape
    if sm_scale is None:
        sm_scale = 1.0 / math.sqrt(d)
    if out is None or lse is None or ws is None:
        out, lse, ws = _attend_outputs(q, out, lse, ws, n_seq, h_kv, stream)
    spot_paged_attend8(q, k_pages, v_pages, k_scale, v_scale, page_table, n_pages, page, max_pages,
                       seq_start, seq_len, n_seq, rows, h_q, h_kv, d, sm_scale, softcap, slopes,
                       window, n_sink, prefix, first, out, lse, ws, stream)
    return out, lse


def paged_weights(q, lse, k_pages, page_table, seq_start, seq_len, sm_scale=None, softcap=0.0,
                  slopes=None, window=0, prefix=None, first=None, acc=None, decay=1.0, out=None,
                  stream=None):
    """Attention weight each cached token received from q, summed per KV head, on top of
    decay * acc: [n_seq, h_kv, max_pages * page_size] float32.  lse from paged_attend (without
    sinks: what those received is left out)."""
    rows, h_q, d = q.shape
    n_pages, h_kv, page, _ = k_pages.shape
    n_seq, max_pages = page_table.shape
    _fits(q, None, None, None, max_pages * page, acc, out, k_pages)
    if sm_scale is None:
        sm_scale = 1.0 / math.sqrt(d)
    if out is None:
        with _on(stream, q.device):
            out = torch.empty((n_seq, h_kv, max_pages * page), dtype=torch.float32, device=q.device)
    spot_paged_weights(q, lse, k_pages, page_table, n_pages, page, max_pages, seq_start, seq_len,
                       n_seq, rows, h_q, h_kv, d, sm_scale, softcap, slopes, window, prefix, first,
                       acc, decay, out, stream)
    return out


def cache_evict(acc, k_pages, v_pages, page_table, seq_len, budget, n_sink, n_recent, k_dst, v_dst,
                dst_table, idx=None, new_len=None, acc_out=None, stream=None):
    """Keeps `budget` tokens of each sequence and KV head (sinks, recent ones and the
    heaviest by acc) and copies them to the pages of dst_table; returns (idx [n_seq,
    h_kv, budget], new_len [n_seq], acc_out [n_seq, h_kv, dst_max_pages * page_size])."""
    n_pages, h_kv, page, d = k_pages.shape
    n_seq, max_pages = page_table.shape
    _fits(None, None, None, None, max_pages * page, acc, None, k_pages, v_pages, k_dst, v_dst)
    dev = k_pages.device
    if idx is None or new_len is None or acc_out is None:
        with _on(stream, dev):
            if idx is None:
                idx = torch.empty((n_seq, h_kv, budget), dtype=torch.int32, device=dev)
            if new_len is None:
                new_len = torch.empty(n_seq, dtype=torch.int32, device=dev)
            if acc_out is None:
                acc_out = torch.empty((n_seq, h_kv, dst_table.shape[1] * page), dtype=torch.float32,
                                      device=dev)
    spot_cache_evict(acc, k_pages, v_pages, page_table, n_pages, page, max_pages, seq_len, n_seq,
                     h_kv, d, budget, n_sink, n_recent, k_dst, v_dst, dst_table, k_dst.shape[0],
                     dst_table.shape[1], idx, new_len, acc_out, acc_out.shape[-1], stream)
    return idx, new_len, acc_out


# ------------------------------------------------------- host helpers
def to_device_bf16(a, device="cuda") -> torch.Tensor:
    """uint16 BF16 bit patterns (numpy) -> torch.bfloat16 device tensor."""
    import numpy as np
    t = torch.from_numpy(np.ascontiguousarray(a).view(np.int16))
    return t.to(device).view(torch.bfloat16)


def bf16_to_float_host(t: torch.Tensor):
    return t.detach().float().cpu().numpy()
