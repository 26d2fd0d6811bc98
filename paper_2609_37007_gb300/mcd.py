"""Thin ctypes binding of libmcd.so (include/mcd.h); argument marshalling only.

Every function has the name of the C entry point it wraps.  Device buffers are torch CUDA
tensors (their data_ptr() is passed through); weights are numpy arrays.  Nothing here
computes any part of the decoding path, and there is no fallback: if the library is
missing, loading it raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import Dict, Optional, Tuple

import numpy as np

from .synth import MCDConfig, OuterConfig

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libmcd.so")
_lib: Optional[ctypes.CDLL] = None

MCD_OK = 0
STATUS_NAMES = {0: "MCD_OK", 1: "MCD_ERR_INVALID_ARG", 2: "MCD_ERR_STATE", 3: "MCD_ERR_CUDA",
                4: "MCD_ERR_OOM", 5: "MCD_ERR_TIMEOUT", 6: "MCD_ERR_WEIGHTS", 7: "MCD_ERR_UNSUPPORTED"}

MAX_CALLS = 16
MAX_ROWS = 8
STATIC_TOPK_MAX_ROWS = 128     # MCD_STATIC_TOPK_MAX_ROWS


class McdConfig(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int32), ("hidden", ctypes.c_int32),
                ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("ffn", ctypes.c_int32),
                ("n_pos", ctypes.c_int32), ("vocab", ctypes.c_int32), ("c0_vocab", ctypes.c_int32),
                ("rms_eps", ctypes.c_float), ("rope_base", ctypes.c_float),
                ("qk_norm", ctypes.c_int32), ("weight_dtype", ctypes.c_int32),
                ("draft_len", ctypes.c_int32), ("top_k", ctypes.c_int32),
                ("temperature", ctypes.c_float), ("draft_mode", ctypes.c_int32),
                ("noise_sigma", ctypes.c_float), ("seed", ctypes.c_uint64), ("max_streams", ctypes.c_int32)]


class McdOuterConfig(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int32), ("hidden", ctypes.c_int32),
                ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("ffn", ctypes.c_int32),
                ("c0_vocab", ctypes.c_int32), ("text_vocab", ctypes.c_int32),
                ("max_tokens", ctypes.c_int32), ("rms_eps", ctypes.c_float),
                ("rope_base", ctypes.c_float), ("qk_norm", ctypes.c_int32),
                ("weight_dtype", ctypes.c_int32), ("top_k", ctypes.c_int32),
                ("temperature", ctypes.c_float), ("seed", ctypes.c_uint64)]


class McdPagedKV(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("layer_stride", ctypes.c_int64), ("page_stride", ctypes.c_int64),
                ("head_stride", ctypes.c_int64), ("token_stride", ctypes.c_int64),
                ("n_layers", ctypes.c_int32), ("n_pages", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32)]


class McdChunks(ctypes.Structure):
    _fields_ = [("table", ctypes.c_void_p), ("cached", ctypes.c_void_p), ("row_start", ctypes.c_void_p),
                ("n_seqs", ctypes.c_int32), ("table_stride", ctypes.c_int32), ("n_rows", ctypes.c_int32),
                ("max_rows", ctypes.c_int32), ("max_tokens", ctypes.c_int32)]


class McdRope(ctypes.Structure):
    _fields_ = [("inv_freq", ctypes.c_void_p), ("scale", ctypes.c_float), ("rot_dim", ctypes.c_int32),
                ("interleaved", ctypes.c_int32)]


CALL_TRACE_DTYPE = np.dtype([("a", "<i4"), ("n_rows", "<i4"), ("pos0", "<i4"), ("n_drafts", "<i4"),
                             ("input_ids", "<i4", 8), ("drafts", "<i4", 8), ("n_acc", "<i4"),
                             ("n_emit", "<i4"), ("emitted", "<i4", 8), ("n_next", "<i4"),
                             ("next_drafts", "<i4", 8), ("draft_row", "<i4"), ("reserved", "<i4", 24)])
assert CALL_TRACE_DTYPE.itemsize == 256

MAX_TREE_NODES = 64            # MCD_MAX_TREE_NODES
MAX_TREE_ROWS = 65             # MCD_MAX_TREE_ROWS
TREE_TRACE_DTYPE = np.dtype([("n_rows", "<i4"), ("row_node", "<i4", MAX_TREE_ROWS),
                             ("row_id", "<i4", MAX_TREE_ROWS), ("path_len", "<i4"), ("path", "<i4", 8),
                             ("draft_row", "<i4"), ("n_next", "<i4"), ("next_cand", "<i4", (8, 8)),
                             ("n_passes", "<i4"), ("reserved", "<i4", 17)])
assert TREE_TRACE_DTYPE.itemsize == 896


class MCDError(RuntimeError):
    def __init__(self, fn: str, status: int):
        self.status = status
        super().__init__(f"{fn} failed: {STATUS_NAMES.get(status, status)}")


def library_path() -> str:
    return _LIB_PATH


def load_library() -> ctypes.CDLL:
    """Load the in-tree libmcd.so (built by __graft_entry__.build()); raises if absent."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise RuntimeError(f"{_LIB_PATH} is missing: build it with __graft_entry__.build()")
    lib = ctypes.CDLL(_LIB_PATH)
    P, I32, I64, U32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_uint32
    sig = {
        "mcd_create": (I32, [ctypes.POINTER(McdConfig), P, ctypes.POINTER(P)]),
        "mcd_load_weights": (I32, [P, I32, ctypes.POINTER(ctypes.c_char_p), ctypes.POINTER(P),
                                   ctypes.POINTER(I64)]),
        "mcd_decode_frame": (I32, [P, U32, U32, P, P, P, P, P]),
        "mcd_decode_frame_host": (I32, [P, U32, U32, P, P, P, P, P]),
        "mcd_decode_frames": (I32, [P, I32, P, P, P, P, P, P, P]),
        "mcd_begin_frame": (I32, [P, U32, U32, P, P, P]),
        "mcd_verify_accept": (I32, [P, P, P, P]),
        "mcd_draft": (I32, [P, I32, I32, P, P, P, P, P]),
        "mcd_accept_from_logits": (I32, [P, I32, I32, I32, P, P, P, P, P]),
        "mcd_topk_softmax": (I32, [P, I32, P, P, P, P]),
        "mcd_topk_softmax_static": (I32, [I32, I32, I32, ctypes.c_float, P, P, P, P, P]),
        "mcd_trace_bytes": (I64, [P]),
        "mcd_set_trace": (I32, [P, P]),
        "mcd_set_timeline": (I32, [P, P]),
        "mcd_sync": (I32, [P]),
        "mcd_test_bounded_wait": (I32, [P, I32, ctypes.c_uint64, P]),
        "mcd_call_weight_bytes": (I64, [P, I32]),
        "mcd_num_ctas": (I32, [P]),
        "mcd_destroy": (None, [P]),
        "mcd_status_str": (ctypes.c_char_p, [I32]),
        "mcd_set_tree": (I32, [P, I32, P, P]),
        "mcd_outer_create": (I32, [ctypes.POINTER(McdOuterConfig), P, ctypes.POINTER(P)]),
        "mcd_outer_destroy": (None, [P]),
        "mcd_outer_load_weights": (I32, [P, I32, ctypes.POINTER(ctypes.c_char_p), ctypes.POINTER(P),
                                         ctypes.POINTER(I64)]),
        "mcd_outer_prefill": (I32, [P, U32, I32, P, P]),
        "mcd_outer_step": (I32, [P, P, I32, P]),
        "mcd_outer_frame_inputs": (I32, [P, ctypes.POINTER(P), ctypes.POINTER(P), ctypes.POINTER(P),
                                         ctypes.POINTER(U32)]),
        "mcd_pipeline_frames": (I32, [P, I32, P, P, P]),
        "mcd_outer_trace_floats": (I64, [P]),
        "mcd_outer_set_trace": (I32, [P, P, I32]),
        "mcd_outer_sync": (I32, [P]),
        "mcd_outer_step_weight_bytes": (I64, [P]),
        "mcd_tc_gemm": (I32, [I32, I32, I32, I32, P, P, P, P]),
        "mcd_tc_tile": (I32, [I32, I32, I32, P, P, P]),
        "mcd_tc_gemm_tiled": (I32, [I32, I32, I32, I32, P, P, P, P, P]),
        "mcd_rope_freqs": (I32, [I32, I32, ctypes.c_double, ctypes.c_double, I32, ctypes.c_double, ctypes.c_double,
                                 P, P]),
        "mcd_rope_append": (I32, [P, I32, P, I32, P, I64, I32, P, I64, P, P, P, P, ctypes.c_float, P, P]),
        "mcd_paged_attention": (I32, [P, I32, P, I32, P, I64, P, I64, ctypes.c_float, P, I32, P, I64, P, P]),
        "mcd_paged_attention_workspace": (I64, [P, P, I32]),
        "mcd_pages_fork": (I32, [P, P, P, I32, P, I32, P, I32, P, P, P, I32, P, I32, P, I64, P, P]),
        "mcd_pages_fork_workspace": (I64, [I32, I32, I32]),
        "mcd_pages_compact": (I32, [P, I32, P, P, I32, P, P, I32, P, P, P, P]),
    }
    for name, (res, args) in sig.items():
        f = getattr(lib, name)
        f.restype = res
        f.argtypes = args
    _lib = lib
    return lib


def _check(fn: str, status: int):
    if status != MCD_OK:
        raise MCDError(fn, status)


def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("device buffers must be CUDA tensors")
    return t.data_ptr()


def _hptr(a) -> Optional[int]:
    """Host buffer address: a C-contiguous numpy array or CPU torch tensor."""
    if a is None:
        return None
    if isinstance(a, np.ndarray):
        if not a.flags["C_CONTIGUOUS"]:
            raise ValueError("host buffers must be C-contiguous")
        return a.ctypes.data
    if a.is_cuda or not a.is_contiguous():
        raise ValueError("host buffers must be contiguous CPU tensors")
    return a.data_ptr()


def config_struct(cfg: MCDConfig) -> McdConfig:
    return McdConfig(cfg.n_layers, cfg.hidden, cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim, cfg.ffn,
                     cfg.n_pos, cfg.vocab, cfg.c0_vocab, cfg.rms_eps, cfg.rope_base, cfg.qk_norm,
                     cfg.weight_dtype, cfg.draft_len, cfg.top_k, cfg.temperature, cfg.draft_mode,
                     cfg.noise_sigma, cfg.sample_seed, cfg.max_streams)


# ---- one wrapper per entry point ------------------------------------------------------
def mcd_create(cfg: MCDConfig, stream=None) -> ctypes.c_void_p:
    lib = load_library()
    c = config_struct(cfg)
    out = ctypes.c_void_p()
    s = ctypes.c_void_p(stream.cuda_stream if stream is not None else None)
    _check("mcd_create", lib.mcd_create(ctypes.byref(c), s, ctypes.byref(out)))
    return out


def _weight_args(weights: Dict[str, np.ndarray]):
    names = list(weights)
    arrs = [np.ascontiguousarray(weights[k]) for k in names]
    n = len(names)
    c_names = (ctypes.c_char_p * n)(*[k.encode() for k in names])
    c_ptrs = (ctypes.c_void_p * n)(*[a.ctypes.data for a in arrs])
    c_sz = (ctypes.c_int64 * n)(*[a.nbytes for a in arrs])
    return n, c_names, c_ptrs, c_sz, arrs


def mcd_load_weights(ctx, weights: Dict[str, np.ndarray]):
    n, c_names, c_ptrs, c_sz, _keep = _weight_args(weights)
    _check("mcd_load_weights", load_library().mcd_load_weights(ctx, n, c_names, c_ptrs, c_sz))


def mcd_decode_frame(ctx, stream_id: int, frame_idx: int, cond, c0, c0_emb, codes_out, stats=None):
    _check("mcd_decode_frame", load_library().mcd_decode_frame(
        ctx, stream_id, frame_idx, _ptr(cond), _ptr(c0), _ptr(c0_emb), _ptr(codes_out), _ptr(stats)))


def mcd_decode_frames(ctx, stream_ids, frame_idx, cond, c0, c0_emb, codes_out, stats=None):
    """Several streams' frames in one launch; stream_ids / frame_idx are host integer lists."""
    n = len(stream_ids)
    sid = (ctypes.c_uint32 * n)(*[int(v) for v in stream_ids])
    fid = (ctypes.c_uint32 * n)(*[int(v) for v in frame_idx])
    _check("mcd_decode_frames", load_library().mcd_decode_frames(
        ctx, n, sid, fid, _ptr(cond), _ptr(c0), _ptr(c0_emb), _ptr(codes_out), _ptr(stats)))


def mcd_decode_frame_host(ctx, stream_id: int, frame_idx: int, cond, c0, c0_emb, codes_out, stats=None):
    """Host buffers (numpy arrays or CPU tensors, pinned or pageable); returns when done."""
    _check("mcd_decode_frame_host", load_library().mcd_decode_frame_host(
        ctx, stream_id, frame_idx, _hptr(cond), _hptr(c0), _hptr(c0_emb), _hptr(codes_out), _hptr(stats)))


def mcd_begin_frame(ctx, stream_id: int, frame_idx: int, cond, c0, c0_emb):
    _check("mcd_begin_frame", load_library().mcd_begin_frame(
        ctx, stream_id, frame_idx, _ptr(cond), _ptr(c0), _ptr(c0_emb)))


def mcd_verify_accept(ctx, emitted, n_emitted, logits_out=None):
    _check("mcd_verify_accept", load_library().mcd_verify_accept(
        ctx, _ptr(emitted), _ptr(n_emitted), _ptr(logits_out)))


def mcd_draft(ctx, pos_k: int, call_idx: int, h_k, draft_ids, q_ids=None, q_weights=None, z_out=None):
    _check("mcd_draft", load_library().mcd_draft(
        ctx, pos_k, call_idx, _ptr(h_k), _ptr(draft_ids), _ptr(q_ids), _ptr(q_weights), _ptr(z_out)))


def mcd_accept_from_logits(ctx, a: int, n_drafts: int, call_idx: int, p_logits, q_logits, draft_ids,
                           emitted, out2):
    _check("mcd_accept_from_logits", load_library().mcd_accept_from_logits(
        ctx, a, n_drafts, call_idx, _ptr(p_logits), _ptr(q_logits), _ptr(draft_ids), _ptr(emitted),
        _ptr(out2)))


def mcd_topk_softmax(ctx, n_rows: int, logits, ids, weights=None, sums=None):
    _check("mcd_topk_softmax", load_library().mcd_topk_softmax(ctx, n_rows, _ptr(logits), _ptr(ids),
                                                                _ptr(weights), _ptr(sums)))


def mcd_topk_softmax_static(n_rows: int, vocab: int, top_k: int, temperature: float, logits, ids,
                            weights=None, sums=None, stream=None):
    _check("mcd_topk_softmax_static", load_library().mcd_topk_softmax_static(
        n_rows, vocab, top_k, temperature, _ptr(logits), _ptr(ids), _ptr(weights), _ptr(sums),
        ctypes.c_void_p(stream.cuda_stream if stream is not None else None)))


def mcd_trace_bytes(ctx) -> int:
    return int(load_library().mcd_trace_bytes(ctx))


def mcd_set_trace(ctx, trace):
    _check("mcd_set_trace", load_library().mcd_set_trace(ctx, _ptr(trace)))


def mcd_set_timeline(ctx, timeline):
    _check("mcd_set_timeline", load_library().mcd_set_timeline(ctx, _ptr(timeline)))


def mcd_sync(ctx):
    _check("mcd_sync", load_library().mcd_sync(ctx))


def mcd_test_bounded_wait(ctx, kind: int, wait_ns: int) -> Tuple[int, int]:
    """(status, device-measured wait in ns) of one bounded wait on something nothing
    signals; MCD_ERR_TIMEOUT is the expected status."""
    waited = ctypes.c_uint64(0)
    st = int(load_library().mcd_test_bounded_wait(ctx, kind, wait_ns, ctypes.addressof(waited)))
    return st, int(waited.value)


def mcd_call_weight_bytes(ctx, n_heads: int) -> int:
    return int(load_library().mcd_call_weight_bytes(ctx, n_heads))


def mcd_num_ctas(ctx) -> int:
    return int(load_library().mcd_num_ctas(ctx))


def mcd_destroy(ctx):
    load_library().mcd_destroy(ctx)


def mcd_tc_gemm(M: int, N: int, K: int, bn: int, A, B, Y, stream=None):
    """Y[n][m] = sum_k A[m][k] B[n][k] on the tensor cores (tcgen05): A bf16 [M, K], B bf16
    [N, K], Y fp32 [N, M], all device tensors (synchronises the stream)."""
    _check("mcd_tc_gemm", load_library().mcd_tc_gemm(M, N, K, bn, _ptr(A), _ptr(B), _ptr(Y),
                                                     ctypes.c_void_p(stream.cuda_stream if stream is not None else None)))


def mcd_tc_tile(R: int, K: int, src, dst, stream=None, ld=None):
    """Re-lay device bf16 src [R][K] (row stride ld, default K) into the swizzled tile layout
    of mcd_tc_gemm_tiled in dst (device, R * K * 2 bytes); asynchronous on the stream."""
    _check("mcd_tc_tile", load_library().mcd_tc_tile(R, K, K if ld is None else ld, _ptr(src), _ptr(dst),
                                                     ctypes.c_void_p(stream.cuda_stream if stream is not None else None)))


def mcd_tc_gemm_tiled(M: int, N: int, K: int, bn: int, A_tiled, B_tiled, Y, err, stream=None):
    """Y[n][m] = sum_k A[m][k] B[n][k] from tiled operands (mcd_tc_tile); err: device int32,
    zeroed by the caller.  Asynchronous: launches the product on the stream and returns."""
    _check("mcd_tc_gemm_tiled", load_library().mcd_tc_gemm_tiled(
        M, N, K, bn, _ptr(A_tiled), _ptr(B_tiled), _ptr(Y), _ptr(err),
        ctypes.c_void_p(stream.cuda_stream if stream is not None else None)))


# ---- paged cache (include/mcd_cache.h) ---------------------------------------------------
# These calls are short, so that their checks of arguments are too: no helper call per property, descriptors carry
# their address, torch's types are looked up once.  A loop keeps its descriptors and workspaces while buffers and bounds
# stay (lengths are read on the device): attention of one row over 630 keys takes 7.3 us a call then, 15.3 with a chunks
# descriptor, its workspace query and the workspace made anew for each.
ROPE_PLAIN, ROPE_LINEAR, ROPE_BASE, ROPE_BY_PARTS = 0, 1, 2, 3
_F32 = _BF16 = _I32 = _F64 = None


def _types():
    """torch's types, once a descriptor is built (the module itself does without torch)."""
    global _F32, _BF16, _I32, _F64
    if _F32 is None:
        import torch
        _F32, _BF16, _I32, _F64 = torch.float32, torch.bfloat16, torch.int32, torch.float64


def _kv_dtype(t) -> int:
    if t.dtype is _F32:
        return 0                    # MCD_WEIGHT_F32
    if t.dtype is _BF16:
        return 1                    # MCD_WEIGHT_BF16
    raise ValueError("rows and pages are float32 or bfloat16")


def _i32(t, what: str, n: int = -1) -> Optional[int]:
    """Address of a contiguous int32 device tensor (of n elements, where given)."""
    if t is None:
        return None
    if t.dtype is not _I32 or not t.is_contiguous() or not t.is_cuda or (n >= 0 and t.numel() != n):
        raise ValueError(f"{what}: a contiguous int32 CUDA tensor" + ("" if n < 0 else f" of {n} elements"))
    return t.data_ptr()


def _gain(t, n: int) -> Optional[int]:
    if t is None:
        return None
    if t.dtype is not _F32 or t.numel() != n or not t.is_contiguous() or not t.is_cuda:
        raise ValueError(f"norm gains: {n} contiguous float32 values on the device")
    return t.data_ptr()


def _rows(t, what: str, n_rows: int, width: int) -> int:
    """Row stride (elements) of a packed device row buffer whose rows hold `width` contiguous elements."""
    n = len(t)
    if not t.is_cuda:
        raise ValueError(f"{what}: device buffers must be CUDA tensors")
    if t.is_contiguous():
        row = stride = t.numel() // n if n else 0
    else:
        row, stride = 1, t.stride(0)
        for size, st in zip(reversed(t.shape[1:]), reversed(t.stride()[1:])):
            if size != 1 and st != row:
                raise ValueError(f"{what}: a row's elements are contiguous")
            row *= size
    if n_rows and (n < n_rows or row < width):
        raise ValueError(f"{what}: at least {n_rows} rows of {width} elements")
    return max(stride, row) if n < 2 else stride


def _space(t) -> Tuple[Optional[int], int]:
    return (None, 0) if t is None else (_ptr(t), t.nbytes)


def paged_kv(k, v) -> McdPagedKV:
    """Descriptor of a page pool: k and v device tensors [layers, pages, kv heads, page size, head dim]
    (float32 or bfloat16) of the same shape and strides, the last dimension contiguous.  It keeps them."""
    _types()
    if k.dim() != 5 or k.shape != v.shape or k.dtype != v.dtype or k.stride() != v.stride() or k.stride(4) != 1:
        raise ValueError("k and v: [layers, pages, kv heads, page size, head dim] alike, the last dimension contiguous")
    st = k.stride()
    d = McdPagedKV(_ptr(k), _ptr(v), st[0], st[1], st[2], st[3], *k.shape, _kv_dtype(k))
    d.kept, d.addr, d.type = (k, v), ctypes.addressof(d), k.dtype
    return d


def chunks(table, cached, row_start, n_rows: int, max_rows: int, max_tokens: int) -> McdChunks:
    """Descriptor of a call's new rows: table int32 [sequences, columns], cached int32 [sequences], row_start
    int32 [sequences + 1], all on the device; the rest are host bounds.  It keeps them."""
    _types()
    n = cached.numel()
    if table.dim() != 2 or table.shape[0] != n:
        raise ValueError("table: [sequences, columns]")
    d = McdChunks(_i32(table, "table"), _i32(cached, "cached"), _i32(row_start, "row_start", n + 1), n, table.shape[1], n_rows,
                  max_rows, max_tokens)
    d.kept, d.addr = (table, cached, row_start), ctypes.addressof(d)
    return d


def rope(inv_freq=None, rot_dim: int = 0, interleaved: bool = False, scale: float = 1.0) -> McdRope:
    """Descriptor of a rotation: inv_freq float64 [rot_dim / 2] on the device; rot_dim 0: none."""
    _types()
    if rot_dim and (inv_freq.dtype is not _F64 or not inv_freq.is_contiguous() or inv_freq.numel() != rot_dim // 2):
        raise ValueError("inv_freq: rot_dim / 2 contiguous float64 values")
    d = McdRope(_ptr(inv_freq) if rot_dim else None, scale, rot_dim, int(interleaved))
    d.kept, d.addr = inv_freq, ctypes.addressof(d)
    return d


def mcd_rope_freqs(rot_dim: int, base: float, kind: int = ROPE_PLAIN, factor: float = 1.0, train_tokens: int = 0,
                   beta_fast: float = 32.0, beta_slow: float = 1.0) -> Tuple[np.ndarray, float]:
    """(frequencies float64 [rot_dim / 2], scale) of the named kind; on the host."""
    out = np.zeros(max(rot_dim // 2, 1), dtype=np.float64)
    scale = ctypes.c_float()
    _check("mcd_rope_freqs", load_library().mcd_rope_freqs(kind, rot_dim, base, factor, train_tokens, beta_fast,
                                                           beta_slow, out.ctypes.data, ctypes.addressof(scale)))
    return out, float(scale.value)


def mcd_rope_append(kv: McdPagedKV, layer: int, ch: McdChunks, n_q_heads: int, qkv, q_out, rot: McdRope, err,
                    positions=None, q_norm=None, k_norm=None, eps: float = 1e-6, stream=None):
    """New rows' q | k | v (qkv [rows, (q + 2 kv heads) * head dim]) normalised, rotated, written to q_out
    [rows, q heads * head dim] (the cache's type) and to the pages of `layer`; asynchronous."""
    d, n = kv.head_dim, ch.n_rows
    if q_out.dtype is not kv.type:
        raise ValueError("q_out has the cache's type")
    st = (_lib or load_library()).mcd_rope_append(
        kv.addr, layer, ch.addr, n_q_heads, qkv.data_ptr(), _rows(qkv, "qkv", n, (n_q_heads + 2 * kv.n_kv_heads) * d), _kv_dtype(qkv),
        q_out.data_ptr(), _rows(q_out, "q_out", n, n_q_heads * d), rot.addr,
        None if positions is None else _i32(positions, "positions", n), None if q_norm is None else _gain(q_norm, d),
        None if k_norm is None else _gain(k_norm, d), eps, _i32(err, "err"), None if stream is None else stream.cuda_stream)
    if st:
        _check("mcd_rope_append", st)


def mcd_paged_attention_workspace(kv: McdPagedKV, ch: McdChunks, n_q_heads: int) -> int:
    return int(load_library().mcd_paged_attention_workspace(kv.addr, ch.addr, n_q_heads))


def mcd_paged_attention(kv: McdPagedKV, layer: int, ch: McdChunks, n_q_heads: int, q, out, scale: float, workspace, err,
                        mask=None, stream=None):
    """out [rows, q heads * head dim] = attention of the new rows q over the pages of `layer`, causal, or among the new
    rows as the bits of mask (int32 [rows, words]) say; workspace: uint8, mcd_paged_attention_workspace
    bytes, or None where that is 0.  Asynchronous."""
    w, n = n_q_heads * kv.head_dim, ch.n_rows
    if q.dtype is not kv.type or out.dtype is not kv.type:
        raise ValueError("q and out have the cache's type")
    words = 0
    if mask is not None:
        if mask.dim() != 2 or mask.shape[0] < n:
            raise ValueError("mask: [rows, words]")
        words = mask.shape[1]
    space, size = _space(workspace)
    st = (_lib or load_library()).mcd_paged_attention(
        kv.addr, layer, ch.addr, n_q_heads, q.data_ptr(), _rows(q, "q", n, w), out.data_ptr(), _rows(out, "out", n, w), scale,
        None if mask is None else _i32(mask, "mask"), words, space, size, _i32(err, "err"),
        None if stream is None else stream.cuda_stream)
    if st:
        _check("mcd_paged_attention", st)


def mcd_pages_fork_workspace(n_src: int, table_out) -> int:
    return int(load_library().mcd_pages_fork_workspace(n_src, *table_out.shape))


def mcd_pages_fork(kv: McdPagedKV, ref_in, ref_out, table_in, len_in, parent, table_out, len_out, workspace, err,
                   reserve=None, release: bool = False, stream=None):
    """Sequences of table_out from those of table_in (int32 device tensors throughout); asynchronous."""
    n_src, src_cols = table_in.shape
    n_dst, dst_cols = table_out.shape
    n_pages = kv.n_pages
    space, size = _space(workspace)
    st = (_lib or load_library()).mcd_pages_fork(
        kv.addr, _i32(ref_in, "ref_in", n_pages), _i32(ref_out, "ref_out", n_pages), n_src, _i32(table_in, "table_in"), src_cols,
        _i32(len_in, "len_in", n_src), n_dst, _i32(parent, "parent", n_dst), None if reserve is None else _i32(reserve, "reserve", n_dst),
        _i32(table_out, "table_out"), dst_cols, _i32(len_out, "len_out", n_dst), int(release), space, size, _i32(err, "err"),
        None if stream is None else stream.cuda_stream)
    if st:
        _check("mcd_pages_fork", st)


def mcd_pages_compact(kv: McdPagedKV, table_in, table_out, start, keep, n_keep, len_out, err, stream=None):
    """Kept tokens of every sequence moved together, in all layers (int32 device tensors throughout; len_out: a tensor
    of its own that overlaps no other, or None); asynchronous."""
    n, cols = table_in.shape
    if keep.dim() != 2 or len(keep) != n:
        raise ValueError("keep: [sequences, most kept]")
    st = (_lib or load_library()).mcd_pages_compact(
        kv.addr, n, _i32(table_in, "table_in"), _i32(table_out, "table_out", n * cols), cols, _i32(start, "start", n), _i32(keep, "keep"),
        keep.shape[1], _i32(n_keep, "n_keep", n), None if len_out is None else _i32(len_out, "len_out", n), _i32(err, "err"),
        None if stream is None else stream.cuda_stream)
    if st:
        _check("mcd_pages_compact", st)


def mcd_status_str(status: int) -> str:
    return load_library().mcd_status_str(status).decode()


def parse_trace(buf: np.ndarray, vocab: int):
    """Split a trace buffer (uint8, mcd_trace_bytes long) into (records, verify, draft)."""
    rec_bytes = CALL_TRACE_DTYPE.itemsize * MAX_CALLS
    recs = buf[:rec_bytes].view(CALL_TRACE_DTYPE)
    logits = buf[rec_bytes:].view(np.float32)
    n = MAX_CALLS * MAX_ROWS * vocab
    return recs, logits[:n].reshape(MAX_CALLS, MAX_ROWS, vocab), logits[n:2 * n].reshape(
        MAX_CALLS, MAX_ROWS, vocab)


def mcd_set_tree(ctx, parent, rank):
    """Sparse tree of TREE mode: parent[i] (-1: child of the call's first row), rank[i]."""
    n = len(parent)
    pa = (ctypes.c_int32 * n)(*[int(v) for v in parent])
    rk = (ctypes.c_int32 * n)(*[int(v) for v in rank])
    _check("mcd_set_tree", load_library().mcd_set_tree(ctx, n, pa, rk))


def parse_tree_trace(buf: np.ndarray, vocab: int):
    """TREE mode: (tree records [16], verify logits of every row [16 calls][65 rows][vocab])."""
    start = CALL_TRACE_DTYPE.itemsize * MAX_CALLS + 2 * MAX_CALLS * MAX_ROWS * vocab * 4
    n = TREE_TRACE_DTYPE.itemsize * MAX_CALLS
    recs = buf[start:start + n].view(TREE_TRACE_DTYPE)
    nv = MAX_CALLS * MAX_TREE_ROWS * vocab
    vall = buf[start + n:start + n + nv * 4].view(np.float32).reshape(MAX_CALLS, MAX_TREE_ROWS, vocab)
    return recs, vall


class Decoder:
    """Owns one context: weights, per-frame state and the stream it runs on."""

    def __init__(self, cfg: MCDConfig, weights: Optional[Dict[str, np.ndarray]] = None, stream=None):
        import torch
        self.cfg = cfg
        self.stream = stream if stream is not None else torch.cuda.current_stream()
        self.ctx = mcd_create(cfg, self.stream)
        if weights is not None:
            mcd_load_weights(self.ctx, weights)

    def close(self):
        if self.ctx:
            mcd_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ---- outer CodeDecoder and the frame pipeline (include/mcd_pipeline.h) ------------------
def outer_config_struct(cfg: OuterConfig) -> McdOuterConfig:
    return McdOuterConfig(cfg.n_layers, cfg.hidden, cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim, cfg.ffn,
                          cfg.c0_vocab, cfg.text_vocab, cfg.max_tokens, cfg.rms_eps, cfg.rope_base,
                          cfg.qk_norm, cfg.weight_dtype, cfg.top_k, cfg.temperature, cfg.sample_seed)


def mcd_outer_create(cfg: OuterConfig, inner_ctx) -> ctypes.c_void_p:
    c = outer_config_struct(cfg)
    out = ctypes.c_void_p()
    _check("mcd_outer_create", load_library().mcd_outer_create(ctypes.byref(c), inner_ctx, ctypes.byref(out)))
    return out


def mcd_outer_destroy(o):
    load_library().mcd_outer_destroy(o)


def mcd_outer_load_weights(o, weights: Dict[str, np.ndarray]):
    n, c_names, c_ptrs, c_sz, _keep = _weight_args(weights)
    _check("mcd_outer_load_weights", load_library().mcd_outer_load_weights(o, n, c_names, c_ptrs, c_sz))


def mcd_outer_prefill(o, stream_id: int, text_ids, c0_out=None):
    _check("mcd_outer_prefill", load_library().mcd_outer_prefill(o, stream_id, int(text_ids.numel()),
                                                                  _ptr(text_ids), _ptr(c0_out)))


def mcd_outer_step(o, prev_codes, text_id: int = -1, c0_out=None):
    _check("mcd_outer_step", load_library().mcd_outer_step(o, _ptr(prev_codes), int(text_id), _ptr(c0_out)))


def mcd_outer_frame_inputs(o):
    """Device addresses (cond, c0_emb, c0) and the frame index of the current frame."""
    cond, emb, c0 = ctypes.c_void_p(), ctypes.c_void_p(), ctypes.c_void_p()
    fi = ctypes.c_uint32()
    _check("mcd_outer_frame_inputs", load_library().mcd_outer_frame_inputs(
        o, ctypes.byref(cond), ctypes.byref(emb), ctypes.byref(c0), ctypes.byref(fi)))
    return cond.value, emb.value, c0.value, fi.value


def mcd_pipeline_frames(o, n_frames: int, codes_out, text_ids=None, stats=None):
    tid = None
    if text_ids is not None:
        tid = (ctypes.c_int32 * n_frames)(*[int(v) for v in text_ids])
    _check("mcd_pipeline_frames", load_library().mcd_pipeline_frames(o, n_frames, tid, _ptr(codes_out),
                                                                      _ptr(stats)))


def mcd_outer_trace_floats(o) -> int:
    return int(load_library().mcd_outer_trace_floats(o))


def mcd_outer_set_trace(o, trace, n_frames: int):
    _check("mcd_outer_set_trace", load_library().mcd_outer_set_trace(o, _ptr(trace), n_frames))


def mcd_outer_sync(o):
    _check("mcd_outer_sync", load_library().mcd_outer_sync(o))


def mcd_outer_step_weight_bytes(o) -> int:
    return int(load_library().mcd_outer_step_weight_bytes(o))


class Pipeline:
    """An inner Decoder plus the outer CodeDecoder on top of it (one utterance at a time)."""

    def __init__(self, outer_cfg: OuterConfig, inner_cfg: MCDConfig,
                 outer_weights: Optional[Dict[str, np.ndarray]] = None,
                 inner_weights: Optional[Dict[str, np.ndarray]] = None, stream=None):
        self.inner = Decoder(inner_cfg, inner_weights, stream)
        self.cfg = outer_cfg
        self.o = mcd_outer_create(outer_cfg, self.inner.ctx)
        if outer_weights is not None:
            mcd_outer_load_weights(self.o, outer_weights)

    def close(self):
        if self.o:
            mcd_outer_destroy(self.o)
            self.o = None
        self.inner.close()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
