"""Thin ctypes binding over liba2ats.so (the C ABI in include/a2ats.h).

Argument marshalling only: every step of the path runs in the HIP kernels.  PyTorch is
used for device memory and for the current HIP stream.  There is no CPU fallback: if
the library is missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liba2ats.so")

F32, BF16 = 0, 1
W_NONE, W_DIAG, W_BLOCK = 0, 1, 2
W_PREPARED = 0x100
OP_ENCODE, OP_LUT, OP_SCORE_TOPK, OP_ATTN, OP_FIT, OP_SEED, OP_BLOCK_TOPK, OP_ATTN_KV8, OP_ATTN_KV4 = 0, 1, 2, 3, 4, 5, 6, 7, 8
I8, E4M3 = 0, 1
EXPORTS = ["a2ats_version", "a2ats_status_string", "a2ats_lut_elems", "a2ats_workspace_bytes", "a2ats_encode_prepare",
           "a2ats_rope_tables", "a2ats_encode_keys", "a2ats_build_lut", "a2ats_score_topk",
           "a2ats_sparse_attn", "a2ats_score_topk_stats", "a2ats_score_topk_plan", "a2ats_score_topk_profiled",
           "a2ats_decode_prologue", "a2ats_decode_select", "a2ats_build_lut_shared", "a2ats_sparse_attn_shared",
           "a2ats_decode_select_shared",
           "a2ats_second_moment", "a2ats_codebook_update", "a2ats_kmeanspp_seed", "a2ats_sparse_attn_paged",
           "a2ats_sparse_attn_static", "a2ats_score_topk_paged", "a2ats_codes_to_pages",
           "a2ats_sparse_attn_host", "a2ats_kv8_append", "a2ats_key_bounds", "a2ats_block_topk",
           "a2ats_sparse_attn_kv8", "a2ats_kv4_append", "a2ats_kv4_read", "a2ats_sparse_attn_kv4", "a2ats_qk_norm_rope"]


class A2atsError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: status {status} ({status_string(status)})")


class Dims(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("n_sub", ctypes.c_int32), ("sub_dim", ctypes.c_int32),
                ("n_centroids", ctypes.c_int32), ("ctx_len", ctypes.c_int32), ("ctx_stride", ctypes.c_int64)]


class KvBlocksStruct(ctypes.Structure):
    _fields_ = [(x, ctypes.c_void_p) for x in ("k", "v", "k_scale", "v_scale", "k_tail", "v_tail", "bounds", "page_table")] + \
               [(x, ctypes.c_int32) for x in ("page_size", "block", "format", "kv_dtype")]


class Kv4Struct(ctypes.Structure):
    _fields_ = [(x, ctypes.c_void_p) for x in ("rows", "scales", "bounds", "page_table")] + \
               [(x, ctypes.c_int32) for x in ("page_size", "block", "kv_dtype")]


_lib = None


def lib() -> ctypes.CDLL:
    """Load the built library (build it with paper_2502_12665_amd.build.build() first)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(f"{LIB_PATH} is not built; run __graft_entry__.build() "
                                    "or `python -m paper_2502_12665_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
        dp = ctypes.POINTER(Dims)
        L.a2ats_version.restype = ctypes.c_int
        L.a2ats_status_string.restype = ctypes.c_char_p
        L.a2ats_status_string.argtypes = [ctypes.c_int]
        L.a2ats_lut_elems.restype = sz
        L.a2ats_lut_elems.argtypes = [dp]
        L.a2ats_workspace_bytes.restype = sz
        L.a2ats_workspace_bytes.argtypes = [dp, ctypes.c_int, i32, i32]
        L.a2ats_rope_tables.restype = ctypes.c_int
        L.a2ats_rope_tables.argtypes = [i32, vp, i32, i32, vp, vp, vp, vp]
        L.a2ats_encode_keys.restype = ctypes.c_int
        L.a2ats_encode_keys.argtypes = [dp, vp, i32, i32, vp, vp, ctypes.c_int, vp, vp, sz, vp]
        L.a2ats_build_lut.restype = ctypes.c_int
        L.a2ats_encode_prepare.argtypes = [dp, vp, vp, ctypes.c_int, vp, sz, vp]
        L.a2ats_encode_prepare.restype = ctypes.c_int
        L.a2ats_build_lut.argtypes = [dp, vp, ctypes.c_int, vp, vp, vp, vp, vp, vp, vp]
        L.a2ats_decode_prologue.restype = ctypes.c_int
        L.a2ats_decode_prologue.argtypes = [dp, vp, i32, i32, vp, vp, ctypes.c_int, vp, vp, ctypes.c_int, vp,
                                            vp, vp, vp, vp, vp, sz, vp]
        L.a2ats_decode_select.restype = ctypes.c_int
        L.a2ats_decode_select.argtypes = [dp, vp, i32, i32, vp, vp, ctypes.c_int, vp, vp, ctypes.c_int, vp, vp, vp,
                                          vp, vp, i32, i32, i32, vp, vp, vp, vp, vp, sz, vp]
        L.a2ats_decode_select_shared.restype = ctypes.c_int
        L.a2ats_decode_select_shared.argtypes = L.a2ats_decode_select.argtypes
        L.a2ats_score_topk.restype = ctypes.c_int
        L.a2ats_score_topk.argtypes = [dp, vp, vp, vp, i32, i32, i32, vp, vp, vp, vp, vp, vp, sz, vp]
        L.a2ats_sparse_attn.restype = ctypes.c_int
        L.a2ats_sparse_attn.argtypes = [dp, vp, vp, vp, vp, ctypes.c_int, vp, vp, i32, i32, i32, vp, vp,
                                        vp, vp, vp, sz, vp]
        L.a2ats_sparse_attn_static.restype = ctypes.c_int
        L.a2ats_sparse_attn_static.argtypes = [dp, vp, vp, vp, vp, ctypes.c_int, vp, vp, i32, i32, i32, vp, vp,
                                               vp, vp, vp]
        L.a2ats_sparse_attn_shared.restype = ctypes.c_int
        L.a2ats_sparse_attn_shared.argtypes = L.a2ats_sparse_attn.argtypes
        L.a2ats_sparse_attn_paged.restype = ctypes.c_int
        L.a2ats_sparse_attn_paged.argtypes = [dp, vp, vp, vp, vp, ctypes.c_int, vp, i32, vp, vp, i32, i32, i32, vp, vp,
                                              vp, vp, vp, sz, vp]
        L.a2ats_build_lut_shared.restype = ctypes.c_int
        L.a2ats_build_lut_shared.argtypes = L.a2ats_build_lut.argtypes
        L.a2ats_kmeanspp_seed.restype = ctypes.c_int
        L.a2ats_kmeanspp_seed.argtypes = [dp, vp, i32, vp, ctypes.c_int, vp, vp, vp, vp, sz, vp]
        L.a2ats_second_moment.restype = ctypes.c_int
        L.a2ats_second_moment.argtypes = [dp, vp, ctypes.c_int64, vp, vp, sz, vp]
        L.a2ats_codebook_update.restype = ctypes.c_int
        L.a2ats_codebook_update.argtypes = [dp, vp, i32, i32, vp, vp, vp, vp, vp, sz, vp]
        L.a2ats_score_topk_plan.restype = ctypes.c_int
        L.a2ats_score_topk_plan.argtypes = [dp, i32, i32, i32, ctypes.POINTER(ctypes.c_int32)]
        L.a2ats_score_topk_stats.restype = ctypes.c_int
        L.a2ats_score_topk_stats.argtypes = [dp, i32, i32, i32, vp, vp, vp]
        L.a2ats_score_topk_profiled.restype = ctypes.c_int
        L.a2ats_score_topk_profiled.argtypes = L.a2ats_score_topk.argtypes + [vp, vp]
        bp = ctypes.POINTER(KvBlocksStruct)
        L.a2ats_kv8_append.restype = ctypes.c_int
        L.a2ats_kv8_append.argtypes = [dp, bp, vp, vp, i32, vp, vp, vp]
        L.a2ats_key_bounds.restype = ctypes.c_int
        L.a2ats_key_bounds.argtypes = [dp, bp, vp, i32, vp, vp, vp]
        L.a2ats_block_topk.restype = ctypes.c_int
        L.a2ats_block_topk.argtypes = [dp, bp, vp, vp, vp, vp, i32, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.a2ats_sparse_attn_kv8.restype = ctypes.c_int
        L.a2ats_sparse_attn_kv8.argtypes = [dp, bp, vp, vp, vp, vp, i32, i32, i32, i32, i32, vp, vp, vp, vp, vp, sz, vp]
        fp = ctypes.POINTER(Kv4Struct)
        L.a2ats_kv4_append.restype = ctypes.c_int
        L.a2ats_kv4_append.argtypes = [dp, fp, vp, vp, i32, vp, vp, vp]
        L.a2ats_kv4_read.restype = ctypes.c_int
        L.a2ats_kv4_read.argtypes = [dp, fp, i32, vp, vp, vp, vp, ctypes.c_int, vp]
        L.a2ats_sparse_attn_kv4.restype = ctypes.c_int
        L.a2ats_sparse_attn_kv4.argtypes = [dp, fp, vp, vp, vp, vp, i32, i32, i32, i32, i32, vp, vp, vp, vp, vp, sz, vp]
        L.a2ats_qk_norm_rope.restype = ctypes.c_int
        L.a2ats_qk_norm_rope.argtypes = [dp, vp, ctypes.c_int64, vp, ctypes.c_int64, ctypes.c_int, i32, vp, vp, ctypes.c_float,
                                         vp, vp, i32, vp, vp, vp, vp, vp, vp, vp]
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().a2ats_status_string(int(status)).decode()


def version() -> int:
    return int(lib().a2ats_version())


def make_dims(batch, n_q_heads, n_kv_heads, head_dim, n_sub, ctx_len, ctx_stride=None,
              n_centroids=256, sub_dim=None) -> Dims:
    return Dims(batch, n_q_heads, n_kv_heads, head_dim, n_sub,
                head_dim // n_sub if sub_dim is None else sub_dim, n_centroids, ctx_len,
                ctx_len if ctx_stride is None else ctx_stride)


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    assert t.is_contiguous(), "tensors crossing the C ABI must be contiguous"
    return ctypes.c_void_p(t.data_ptr())


def host_device_pointer(t: torch.Tensor) -> int:
    """Device-side address of a pinned host tensor (hipHostGetDevicePointer); raises if the memory is
    not mapped into the device's address space.  For caches kept in host memory and read by the GPU
    over PCIe."""
    assert t.device.type == "cpu" and t.is_pinned() and t.is_contiguous()
    hip = ctypes.CDLL("libamdhip64.so")
    hip.hipHostGetDevicePointer.restype = ctypes.c_int
    hip.hipHostGetDevicePointer.argtypes = [ctypes.POINTER(ctypes.c_void_p), ctypes.c_void_p, ctypes.c_uint]
    dev = ctypes.c_void_p()
    rc = hip.hipHostGetDevicePointer(ctypes.byref(dev), ctypes.c_void_p(t.data_ptr()), 0)
    if rc != 0 or not dev.value:
        raise RuntimeError(f"hipHostGetDevicePointer failed ({rc}): the tensor is not mapped for the device")
    return int(dev.value)


def _stream():
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise TypeError(f"unsupported dtype {t.dtype}")


def _check(rc: int, what: str):
    if rc != 0:
        raise A2atsError(rc, what)


def lut_elems(dims: Dims) -> int:
    return int(lib().a2ats_lut_elems(ctypes.byref(dims)))


def workspace_bytes(dims: Dims, op: int, top_k: int = 0, window: int = 0) -> int:
    n = int(lib().a2ats_workspace_bytes(ctypes.byref(dims), op, top_k, window))
    if n == ctypes.c_size_t(-1).value:
        raise A2atsError(-1, "a2ats_workspace_bytes")
    return n


def rope_tables(head_dim: int, inv_freq: torch.Tensor, b: int, window: int, device=None):
    """Host helper -> (cos_b, sin_b [D/2], cos_win, sin_win [window, D/2]) float32, moved to `device`."""
    inv = inv_freq.detach().to("cpu", torch.float64).contiguous()
    half = head_dim // 2
    cb, sb = torch.empty(half, dtype=torch.float32), torch.empty(half, dtype=torch.float32)
    cw = torch.empty(max(window, 1), half, dtype=torch.float32)
    sw = torch.empty(max(window, 1), half, dtype=torch.float32)
    rc = lib().a2ats_rope_tables(head_dim, _ptr(inv), int(b), int(window), _ptr(cb), _ptr(sb), _ptr(cw), _ptr(sw))
    _check(rc, "a2ats_rope_tables")
    outs = (cb, sb, cw, sw)
    return tuple(t.to(device) for t in outs) if device is not None else outs


def encode_keys(dims: Dims, keys, n_new: int, pos0: int, codebook, weights, weight_mode: int, codes,
                ws: Optional[torch.Tensor] = None):
    rc = lib().a2ats_encode_keys(ctypes.byref(dims), _ptr(keys), n_new, pos0, _ptr(codebook), _ptr(weights),
                                 weight_mode, _ptr(codes), _ptr(ws), 0 if ws is None else ws.numel() * ws.element_size(),
                                 _stream())
    _check(rc, "a2ats_encode_keys")


def encode_prepare(dims: Dims, codebook, weights, weight_mode: int, ws: torch.Tensor):
    rc = lib().a2ats_encode_prepare(ctypes.byref(dims), _ptr(codebook), _ptr(weights), weight_mode, _ptr(ws),
                                    ws.numel() * ws.element_size(), _stream())
    _check(rc, "a2ats_encode_prepare")


def build_lut(dims: Dims, q, cos_b, sin_b, codebook, q_rot, lut, lut_scale):
    rc = lib().a2ats_build_lut(ctypes.byref(dims), _ptr(q), _dtype_code(q), _ptr(cos_b), _ptr(sin_b),
                               _ptr(codebook), _ptr(q_rot), _ptr(lut), _ptr(lut_scale), _stream())
    _check(rc, "a2ats_build_lut")


def decode_prologue(dims: Dims, keys, n_new: int, pos0: int, codebook, weights, weight_mode: int, codes,
                    q, cos_b, sin_b, q_rot, lut, lut_scale, ws: Optional[torch.Tensor] = None):
    """encode_keys (the decode-time append of a few keys) and build_lut fused; `ws` for the single codebook."""
    rc = lib().a2ats_decode_prologue(ctypes.byref(dims), _ptr(keys), n_new, pos0, _ptr(codebook),
                                     _ptr(weights), weight_mode, _ptr(codes), _ptr(q), _dtype_code(q),
                                     _ptr(cos_b), _ptr(sin_b), _ptr(q_rot), _ptr(lut), _ptr(lut_scale),
                                     _ptr(ws), 0 if ws is None else ws.numel() * ws.element_size(), _stream())
    _check(rc, "a2ats_decode_prologue")


def decode_select(dims: Dims, keys, n_new: int, pos0: int, codebook, weights, weight_mode: int, codes,
                  q, cos_b, sin_b, q_rot, lut, lut_scale, top_k: int, window: int, n_sink: int, seq_lens,
                  topk_idx, topk_count, topk_score=None, ws: Optional[torch.Tensor] = None):
    """decode_prologue + score_topk as one call (one launch less on the streaming route)."""
    rc = lib().a2ats_decode_select(ctypes.byref(dims), _ptr(keys), n_new, pos0, _ptr(codebook), _ptr(weights),
                                   weight_mode, _ptr(codes), _ptr(q), _dtype_code(q), _ptr(cos_b), _ptr(sin_b),
                                   _ptr(q_rot), _ptr(lut), _ptr(lut_scale), top_k, window, n_sink, _ptr(seq_lens),
                                   _ptr(topk_idx), _ptr(topk_count), _ptr(topk_score), _ptr(ws),
                                   0 if ws is None else ws.numel() * ws.element_size(), _stream())
    _check(rc, "a2ats_decode_select")


def decode_select_shared(dims: Dims, keys, n_new: int, pos0: int, codebook, weights, weight_mode: int, codes,
                         q, cos_b, sin_b, q_rot, lut, lut_scale, top_k: int, window: int, n_sink: int, seq_lens,
                         topk_idx, topk_count, topk_score=None, ws: Optional[torch.Tensor] = None):
    """encode_keys + build_lut_shared + score_topk (one selection per KV head) as one call; `dims` are the
    real ones, lut / lut_scale / topk_* / ws those of dims with n_q_heads = n_kv_heads."""
    rc = lib().a2ats_decode_select_shared(ctypes.byref(dims), _ptr(keys), n_new, pos0, _ptr(codebook),
                                          _ptr(weights), weight_mode, _ptr(codes), _ptr(q), _dtype_code(q),
                                          _ptr(cos_b), _ptr(sin_b), _ptr(q_rot), _ptr(lut), _ptr(lut_scale), top_k,
                                          window, n_sink, _ptr(seq_lens), _ptr(topk_idx), _ptr(topk_count),
                                          _ptr(topk_score), _ptr(ws),
                                          0 if ws is None else ws.numel() * ws.element_size(), _stream())
    _check(rc, "a2ats_decode_select_shared")


def score_topk(dims: Dims, codes, lut, lut_scale, top_k: int, window: int, n_sink: int, seq_lens,
               topk_idx, topk_count, topk_score=None, scores_out=None, ws: Optional[torch.Tensor] = None):
    rc = lib().a2ats_score_topk(ctypes.byref(dims), _ptr(codes), _ptr(lut), _ptr(lut_scale), top_k, window,
                                n_sink, _ptr(seq_lens), _ptr(topk_idx), _ptr(topk_count), _ptr(topk_score),
                                _ptr(scores_out), _ptr(ws), 0 if ws is None else ws.numel() * ws.element_size(),
                                _stream())
    _check(rc, "a2ats_score_topk")


def sparse_attn(dims: Dims, q, q_rot, k_cache, v_cache, topk_idx, topk_count, top_k: int, window: int,
                n_sink: int, cos_win, sin_win, seq_lens, out, ws: Optional[torch.Tensor] = None):
    rc = lib().a2ats_sparse_attn(ctypes.byref(dims), _ptr(q), _ptr(q_rot), _ptr(k_cache), _ptr(v_cache),
                                 _dtype_code(k_cache), _ptr(topk_idx), _ptr(topk_count), top_k, window, n_sink,
                                 _ptr(cos_win), _ptr(sin_win), _ptr(seq_lens), _ptr(out), _ptr(ws),
                                 0 if ws is None else ws.numel() * ws.element_size(), _stream())
    _check(rc, "a2ats_sparse_attn")


def sparse_attn_static(dims: Dims, q, q_rot, k_cache, v_cache, topk_idx, topk_count, top_k: int, window: int,
                       n_sink: int, cos_win, sin_win, seq_lens, out):
    """sparse_attn with its scratch memory inside the library (allocates nothing; at most 8 MiB of it)."""
    rc = lib().a2ats_sparse_attn_static(ctypes.byref(dims), _ptr(q), _ptr(q_rot), _ptr(k_cache), _ptr(v_cache),
                                        _dtype_code(k_cache), _ptr(topk_idx), _ptr(topk_count), top_k, window,
                                        n_sink, _ptr(cos_win), _ptr(sin_win), _ptr(seq_lens), _ptr(out), _stream())
    _check(rc, "a2ats_sparse_attn_static")


def sparse_attn_host(dims: Dims, q, q_rot, k_cache, v_cache, topk_idx, topk_count, top_k: int, window: int,
                     n_sink: int, cos_win, sin_win, seq_lens, out, n_threads: int = 0):
    """sparse_attn on the host CPU over a cache in host memory: every tensor is a CPU tensor."""
    for t in (q, q_rot, k_cache, v_cache, topk_idx, topk_count, cos_win, sin_win, seq_lens, out):
        assert t is None or t.device.type == "cpu", "a2ats_sparse_attn_host takes host pointers"
    rc = lib().a2ats_sparse_attn_host(ctypes.byref(dims), _ptr(q), _ptr(q_rot), _ptr(k_cache), _ptr(v_cache),
                                      _dtype_code(k_cache), _ptr(topk_idx), _ptr(topk_count), top_k, window, n_sink,
                                      _ptr(cos_win), _ptr(sin_win), _ptr(seq_lens), _ptr(out), n_threads)
    _check(rc, "a2ats_sparse_attn_host")


def build_lut_shared(dims: Dims, q, cos_b, sin_b, codebook, q_rot, lut, lut_scale):
    """Tables of one head per KV head from the summed rotated queries of its group (lut / lut_scale
    sized for dims with n_q_heads = n_kv_heads); q_rot per query head."""
    rc = lib().a2ats_build_lut_shared(ctypes.byref(dims), _ptr(q), _dtype_code(q), _ptr(cos_b), _ptr(sin_b),
                                      _ptr(codebook), _ptr(q_rot), _ptr(lut), _ptr(lut_scale), _stream())
    _check(rc, "a2ats_build_lut_shared")


def sparse_attn_shared(dims: Dims, q, q_rot, k_cache, v_cache, topk_idx, topk_count, top_k: int, window: int,
                       n_sink: int, cos_win, sin_win, seq_lens, out, ws: Optional[torch.Tensor] = None):
    """sparse_attn with one selection per KV head (topk_idx [B,Hkv,K], topk_count [B,Hkv])."""
    rc = lib().a2ats_sparse_attn_shared(ctypes.byref(dims), _ptr(q), _ptr(q_rot), _ptr(k_cache), _ptr(v_cache),
                                        _dtype_code(k_cache), _ptr(topk_idx), _ptr(topk_count), top_k, window,
                                        n_sink, _ptr(cos_win), _ptr(sin_win), _ptr(seq_lens), _ptr(out), _ptr(ws),
                                        0 if ws is None else ws.numel() * ws.element_size(), _stream())
    _check(rc, "a2ats_sparse_attn_shared")


def kmeanspp_seed(dims: Dims, keys, n_new: int, weights, weight_mode: int, u, codebook_out, picks, ws: torch.Tensor):
    rc = lib().a2ats_kmeanspp_seed(ctypes.byref(dims), _ptr(keys), n_new, _ptr(weights), weight_mode, _ptr(u),
                                   _ptr(codebook_out), _ptr(picks), _ptr(ws), ws.numel() * ws.element_size(),
                                   _stream())
    _check(rc, "a2ats_kmeanspp_seed")


def second_moment(dims: Dims, q_rot, n_samples: int, h_out, ws: torch.Tensor):
    rc = lib().a2ats_second_moment(ctypes.byref(dims), _ptr(q_rot), n_samples, _ptr(h_out), _ptr(ws),
                                   ws.numel() * ws.element_size(), _stream())
    _check(rc, "a2ats_second_moment")


def codebook_update(dims: Dims, keys, n_new: int, pos0: int, codes, codebook, codebook_out, counts, ws: torch.Tensor):
    rc = lib().a2ats_codebook_update(ctypes.byref(dims), _ptr(keys), n_new, pos0, _ptr(codes), _ptr(codebook),
                                     _ptr(codebook_out), _ptr(counts), _ptr(ws), ws.numel() * ws.element_size(),
                                     _stream())
    _check(rc, "a2ats_codebook_update")


def sparse_attn_paged(dims: Dims, q, q_rot, k_pool, v_pool, page_table, page_size: int, topk_idx, topk_count,
                      top_k: int, window: int, n_sink: int, cos_win, sin_win, seq_lens, out, ws: torch.Tensor):
    """sparse_attn over pools of pages [page][Hkv][page_size][D] addressed through page_table [B, pages]."""
    rc = lib().a2ats_sparse_attn_paged(ctypes.byref(dims), _ptr(q), _ptr(q_rot), _ptr(k_pool), _ptr(v_pool),
                                       _dtype_code(k_pool), _ptr(page_table), page_size, _ptr(topk_idx),
                                       _ptr(topk_count), top_k, window, n_sink, _ptr(cos_win), _ptr(sin_win),
                                       _ptr(seq_lens), _ptr(out), _ptr(ws), ws.numel() * ws.element_size(), _stream())
    _check(rc, "a2ats_sparse_attn_paged")


def score_topk_paged(dims: Dims, code_pool, page_table, page_size: int, lut, lut_scale, top_k: int, window: int,
                     n_sink: int, seq_lens, topk_idx, topk_count, topk_score=None, scores_out=None,
                     ws: Optional[torch.Tensor] = None):
    """score_topk over a pool of code pages [page][Hkv][page_size][M] addressed through page_table [B, pages]."""
    rc = lib().a2ats_score_topk_paged(ctypes.byref(dims), _ptr(code_pool), _ptr(page_table), page_size, _ptr(lut),
                                      _ptr(lut_scale), top_k, window, n_sink, _ptr(seq_lens), _ptr(topk_idx),
                                      _ptr(topk_count), _ptr(topk_score), _ptr(scores_out), _ptr(ws),
                                      0 if ws is None else ws.numel() * ws.element_size(), _stream())
    _check(rc, "a2ats_score_topk_paged")


def codes_to_pages(dims: Dims, new_codes, n_new: int, pos0: int, code_pool, page_table, page_size: int):
    """Copy the code rows [B, Hkv, n_new, M] of freshly encoded tokens to tokens pos0.. of the paged pool."""
    rc = lib().a2ats_codes_to_pages(ctypes.byref(dims), _ptr(new_codes), n_new, pos0, _ptr(code_pool),
                                    _ptr(page_table), page_size, _stream())
    _check(rc, "a2ats_codes_to_pages")


class KvBlocks:
    """A key/value cache cut into blocks of tokens (a2ats_kv_blocks): the tensors and their description, nothing else.

    k, v           int8 or float8_e4m3fn, [B, Hkv, ctx_stride, D], or pages [pages, Hkv, page_size, D]
    k_scale, ...   float32 [.., ctx_stride / block] (pages: page_size / block)
    k_tail, ...    kv_dtype [B, Hkv, block, D]
    bounds         kv_dtype [.., ctx_stride / block, 2, D] (pages: page_size / block)
    All of k .. v_tail are None for a cache of which only the bounds are kept here (key_bounds, block_topk).
    The tensors and their memory stay those that were given: a cache in other memory is another KvBlocks."""

    def __init__(self, dims: Dims, block: int, kv_dtype: torch.dtype, k=None, v=None, k_scale=None, v_scale=None, k_tail=None,
                 v_tail=None, bounds=None, page_table=None, page_size: int = 0):
        rows = (k, v, k_scale, v_scale, k_tail, v_tail)
        if any(t is None for t in rows) != all(t is None for t in rows):
            raise ValueError("k, v, their scales and tails are given together")
        if k is None and bounds is None:
            raise ValueError("neither rows nor bounds")
        _check_blocks(dims, block, kv_dtype, page_table, page_size)
        B, Hkv, D = dims.batch, dims.n_kv_heads, dims.head_dim
        if page_table is not None:
            some = k if k is not None else bounds
            lead = (some.shape[0], Hkv)
            slots = page_size
            _check_tensor(page_table, "page_table", torch.int32, (B, -(-dims.ctx_stride // page_size)))
        else:
            lead, slots = (B, Hkv), int(dims.ctx_stride)
        self.format = I8
        if k is not None:
            if k.dtype not in (torch.int8, torch.float8_e4m3fn):
                raise TypeError(f"codes are int8 or float8_e4m3fn, not {k.dtype}")
            self.format = I8 if k.dtype == torch.int8 else E4M3
            for name, t in (("k", k), ("v", v)):
                _check_tensor(t, name, k.dtype, lead + (slots, D))
            for name, t in (("k_scale", k_scale), ("v_scale", v_scale)):
                _check_tensor(t, name, torch.float32, lead + (slots // block,))
            for name, t in (("k_tail", k_tail), ("v_tail", v_tail)):
                _check_tensor(t, name, kv_dtype, (B, Hkv, block, D))
        if bounds is not None:
            _check_tensor(bounds, "bounds", kv_dtype, lead + (slots // block, 2, D))
        self.block, self.kv_dtype, self.page_size, self.page_table = block, kv_dtype, page_size, page_table
        self.k, self.v, self.k_scale, self.v_scale, self.k_tail, self.v_tail, self.bounds = k, v, k_scale, v_scale, k_tail, v_tail, bounds
        self.device = (k if k is not None else bounds).device
        self.device_index = (k if k is not None else bounds).get_device()
        for t in rows + (bounds, page_table):
            if t is not None and t.device != self.device:
                raise ValueError("the tensors of a cache are on one device")
        p = [None if t is None else t.data_ptr() for t in (k, v, k_scale, v_scale, k_tail, v_tail, bounds, page_table)]
        self.struct = KvBlocksStruct(*p, page_size, block, self.format, F32 if kv_dtype == torch.float32 else BF16)
        self.ref = ctypes.byref(self.struct)
        self.batch, self.n_kv_heads, self.ctx_stride = B, Hkv, int(dims.ctx_stride)

    @classmethod
    def empty(cls, dims: Dims, block: int, kv_dtype: torch.dtype, codes: Optional[torch.dtype] = torch.int8, bounds: bool = True,
              page_table=None, page_size: int = 0, n_pages: int = 0, device="cuda"):
        """A cache in new memory (scales zero).  codes None: only the bounds."""
        _check_blocks(dims, block, kv_dtype, page_table, page_size)
        B, Hkv, D = dims.batch, dims.n_kv_heads, dims.head_dim
        lead, slots = ((n_pages, Hkv), page_size) if page_table is not None else ((B, Hkv), int(dims.ctx_stride))
        t = {}
        if codes is not None:
            for x in ("k", "v"):
                t[x] = torch.empty(lead + (slots, D), dtype=codes, device=device)
                t[x + "_scale"] = torch.zeros(lead + (slots // block,), dtype=torch.float32, device=device)
                t[x + "_tail"] = torch.zeros(B, Hkv, block, D, dtype=kv_dtype, device=device)
        if bounds:
            t["bounds"] = torch.empty(lead + (slots // block, 2, D), dtype=kv_dtype, device=device)
        return cls(dims, block, kv_dtype, page_table=page_table, page_size=page_size, **t)


def _check_blocks(dims: Dims, block: int, kv_dtype: torch.dtype, page_table, page_size: int):
    if kv_dtype not in (torch.float32, torch.bfloat16):
        raise TypeError(f"unsupported dtype {kv_dtype}")
    if block not in (16, 32, 64, 128):
        raise ValueError("block is 16, 32, 64 or 128")
    if page_table is None:
        if dims.ctx_stride % block:
            raise ValueError("ctx_stride is a multiple of block")
    elif page_size < block or page_size & (page_size - 1):
        raise ValueError("page_size is a power of two of at least a block")


def _check_tensor(t: torch.Tensor, name: str, dtype: torch.dtype, shape):
    if t.dtype != dtype:
        raise TypeError(f"{name} is {t.dtype}, not {dtype}")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, not {tuple(shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} is not contiguous")


def _arg(cache: KvBlocks, t: Optional[torch.Tensor], name: str, dtype: torch.dtype, numel: int):
    """Pointer of a tensor of a call on `cache`: of its device, its type and `numel` elements."""
    if t is None:
        return None
    if t.dtype is dtype and t.get_device() == cache.device_index and t.numel() == numel and t.is_contiguous():
        return t.data_ptr()
    if t.dtype != dtype:
        raise TypeError(f"{name} is {t.dtype}, not {dtype}")
    if t.device != cache.device:
        raise ValueError(f"{name} is on {t.device}, the cache on {cache.device}")
    raise ValueError(f"{name}: {numel} contiguous elements are wanted, not {tuple(t.shape)}")


def _cache_stream(dims: Dims, cache: KvBlocks):
    if dims.batch != cache.batch or dims.n_kv_heads != cache.n_kv_heads or dims.ctx_stride != cache.ctx_stride:
        raise ValueError("dims are not those of the cache")
    if cache.device_index < 0:
        raise ValueError(f"the cache is on {cache.device}")
    if cache.device_index != torch.cuda.current_device():
        raise ValueError(f"the cache is on {cache.device}, the current device is {torch.cuda.current_device()}")
    return torch._C._cuda_getCurrentRawStream(cache.device_index)   # current_stream() makes an object of it: 2.8 us


def kv8_append(dims: Dims, cache: KvBlocks, k_new, v_new, n_new: int, seq_lens=None, new_lens=None):
    """Append up to n_new tokens a sequence, k_new / v_new [B, Hkv, n_new, D]; seq_lens count them already, up to dims.ctx_len."""
    B, n = dims.batch, dims.batch * dims.n_kv_heads * n_new * dims.head_dim
    st = _cache_stream(dims, cache)
    rc = lib().a2ats_kv8_append(ctypes.byref(dims), cache.ref, _arg(cache, k_new, "k_new", cache.kv_dtype, n),
                                _arg(cache, v_new, "v_new", cache.kv_dtype, n), n_new,
                                _arg(cache, seq_lens, "seq_lens", torch.int32, B),
                                _arg(cache, new_lens, "new_lens", torch.int32, B), st)
    _check(rc, "a2ats_kv8_append")


def key_bounds(dims: Dims, cache: KvBlocks, k_new, n_new: int, seq_lens=None, new_lens=None):
    """The bounds of the appended tokens' blocks alone."""
    st = _cache_stream(dims, cache)
    rc = lib().a2ats_key_bounds(ctypes.byref(dims), cache.ref,
                                _arg(cache, k_new, "k_new", cache.kv_dtype, dims.batch * dims.n_kv_heads * n_new * dims.head_dim),
                                n_new, _arg(cache, seq_lens, "seq_lens", torch.int32, dims.batch),
                                _arg(cache, new_lens, "new_lens", torch.int32, dims.batch), st)
    _check(rc, "a2ats_key_bounds")


def block_topk(dims: Dims, cache: KvBlocks, q, cos_b, sin_b, q_rot, shared: bool, top_blocks: int, window: int, n_sink: int,
               seq_lens, block_idx, block_count, block_score=None, token_idx=None, token_count=None,
               ws: Optional[torch.Tensor] = None):
    """Rotate the query and select the top_blocks blocks of each query head (shared: of each KV head)."""
    n_q = dims.batch * dims.n_q_heads * dims.head_dim
    n_h = dims.batch * (dims.n_kv_heads if shared else dims.n_q_heads)
    half = dims.head_dim // 2
    st = _cache_stream(dims, cache)
    rc = lib().a2ats_block_topk(ctypes.byref(dims), cache.ref, _arg(cache, q, "q", cache.kv_dtype, n_q),
                                _arg(cache, cos_b, "cos_b", torch.float32, half), _arg(cache, sin_b, "sin_b", torch.float32, half),
                                _arg(cache, q_rot, "q_rot", torch.float32, n_q), int(shared), top_blocks, window, n_sink,
                                _arg(cache, seq_lens, "seq_lens", torch.int32, dims.batch),
                                _arg(cache, block_idx, "block_idx", torch.int32, n_h * top_blocks),
                                _arg(cache, block_count, "block_count", torch.int32, n_h),
                                _arg(cache, block_score, "block_score", torch.float32, n_h * top_blocks),
                                _arg(cache, token_idx, "token_idx", torch.int32, n_h * top_blocks * cache.block),
                                _arg(cache, token_count, "token_count", torch.int32, n_h), _ws_ptr(cache, ws), _ws_bytes(ws), st)
    _check(rc, "a2ats_block_topk")


def sparse_attn_kv8(dims: Dims, cache: KvBlocks, q, q_rot, sel_idx, sel_count, n_sel: int, sel_size: int, shared: bool,
                    window: int, n_sink: int, cos_win, sin_win, seq_lens, out, ws: Optional[torch.Tensor] = None):
    """Attention over sinks, selection (tokens: sel_size 1, or blocks: sel_size cache.block) and window of an 8-bit cache."""
    n_q = dims.batch * dims.n_q_heads * dims.head_dim
    n_h = dims.batch * (dims.n_kv_heads if shared else dims.n_q_heads)
    n_w = max(window, 1) * (dims.head_dim // 2)
    st = _cache_stream(dims, cache)
    rc = lib().a2ats_sparse_attn_kv8(ctypes.byref(dims), cache.ref, _arg(cache, q, "q", cache.kv_dtype, n_q),
                                     _arg(cache, q_rot, "q_rot", torch.float32, n_q),
                                     _arg(cache, sel_idx, "sel_idx", torch.int32, n_h * n_sel),
                                     _arg(cache, sel_count, "sel_count", torch.int32, n_h), n_sel, sel_size, int(shared), window,
                                     n_sink, _arg(cache, cos_win, "cos_win", torch.float32, n_w),
                                     _arg(cache, sin_win, "sin_win", torch.float32, n_w),
                                     _arg(cache, seq_lens, "seq_lens", torch.int32, dims.batch),
                                     _arg(cache, out, "out", cache.kv_dtype, n_q), _ws_ptr(cache, ws), _ws_bytes(ws), st)
    _check(rc, "a2ats_sparse_attn_kv8")


class Kv4Cache:
    """A key/value cache held in 4 bits (a2ats_kv4): the tensors and their description, nothing else.

    rows      uint8 [B, Hkv, ctx_stride, 128], or pages [pages, Hkv, page_size, 128]: a token's codes, key then value
    scales    uint8 [.., 8]: the exponents of its eight groups
    bounds    kv_dtype [.., ctx_stride / block, 2, D] (pages: page_size / block), or None
    blocks is the KvBlocks of the bounds alone, which key_bounds and block_topk take (None without bounds)."""

    def __init__(self, dims: Dims, block: int, kv_dtype: torch.dtype, rows, scales, bounds=None, page_table=None, page_size: int = 0):
        _check_blocks(dims, block, kv_dtype, page_table, page_size)
        B, Hkv = dims.batch, dims.n_kv_heads
        if page_table is not None:
            lead, slots = (rows.shape[0], Hkv), page_size
            _check_tensor(page_table, "page_table", torch.int32, (B, -(-dims.ctx_stride // page_size)))
        else:
            lead, slots = (B, Hkv), int(dims.ctx_stride)
        _check_tensor(rows, "rows", torch.uint8, lead + (slots, 128))
        _check_tensor(scales, "scales", torch.uint8, lead + (slots, 8))
        if bounds is not None and bounds.shape[0] != lead[0]:
            raise ValueError("bounds and rows have different pages")
        for t in (scales, bounds, page_table):
            if t is not None and t.device != rows.device:
                raise ValueError("the tensors of a cache are on one device")
        self.blocks = None if bounds is None else KvBlocks(dims, block, kv_dtype, bounds=bounds, page_table=page_table, page_size=page_size)
        self.block, self.kv_dtype, self.page_size, self.page_table = block, kv_dtype, page_size, page_table
        self.rows, self.scales, self.bounds = rows, scales, bounds
        self.device, self.device_index = rows.device, rows.get_device()
        p = [None if t is None else t.data_ptr() for t in (rows, scales, bounds, page_table)]
        self.struct = Kv4Struct(*p, page_size, block, F32 if kv_dtype == torch.float32 else BF16)
        self.ref = ctypes.byref(self.struct)
        self.batch, self.n_kv_heads, self.ctx_stride = B, Hkv, int(dims.ctx_stride)

    @classmethod
    def empty(cls, dims: Dims, block: int, kv_dtype: torch.dtype, bounds: bool = True, page_table=None, page_size: int = 0,
              n_pages: int = 0, device="cuda"):
        """A cache in new memory (zeros)."""
        _check_blocks(dims, block, kv_dtype, page_table, page_size)
        lead = (n_pages, dims.n_kv_heads) if page_table is not None else (dims.batch, dims.n_kv_heads)
        slots = page_size if page_table is not None else int(dims.ctx_stride)
        rows = torch.zeros(lead + (slots, 128), dtype=torch.uint8, device=device)
        scales = torch.zeros(lead + (slots, 8), dtype=torch.uint8, device=device)
        bd = torch.empty(lead + (slots // block, 2, dims.head_dim), dtype=kv_dtype, device=device) if bounds else None
        return cls(dims, block, kv_dtype, rows, scales, bd, page_table, page_size)


def kv4_append(dims: Dims, cache: Kv4Cache, k_new, v_new, n_new: int, seq_lens=None, new_lens=None):
    """Append up to n_new tokens a sequence, k_new / v_new [B, Hkv, n_new, D]; seq_lens count them already, up to dims.ctx_len."""
    B, n = dims.batch, dims.batch * dims.n_kv_heads * n_new * dims.head_dim
    st = _cache_stream(dims, cache)
    rc = lib().a2ats_kv4_append(ctypes.byref(dims), cache.ref, _arg(cache, k_new, "k_new", cache.kv_dtype, n),
                                _arg(cache, v_new, "v_new", cache.kv_dtype, n), n_new,
                                _arg(cache, seq_lens, "seq_lens", torch.int32, B),
                                _arg(cache, new_lens, "new_lens", torch.int32, B), st)
    _check(rc, "a2ats_kv4_append")


def kv4_read(dims: Dims, cache: Kv4Cache, n_rows: int, seq_lens, new_lens, k_out, v_out):
    """The last tokens of each sequence (as an append with these lengths wrote them) as float32 or bfloat16, k_out / v_out
    [B, Hkv, n_rows, D] of one type; either may be None."""
    B, n = dims.batch, dims.batch * dims.n_kv_heads * n_rows * dims.head_dim
    some = k_out if k_out is not None else v_out
    if some is None:
        raise ValueError("neither k_out nor v_out")
    st = _cache_stream(dims, cache)
    rc = lib().a2ats_kv4_read(ctypes.byref(dims), cache.ref, n_rows, _arg(cache, seq_lens, "seq_lens", torch.int32, B),
                              _arg(cache, new_lens, "new_lens", torch.int32, B), _arg(cache, k_out, "k_out", some.dtype, n),
                              _arg(cache, v_out, "v_out", some.dtype, n), _dtype_code(some), st)
    _check(rc, "a2ats_kv4_read")


def sparse_attn_kv4(dims: Dims, cache: Kv4Cache, q, q_rot, sel_idx, sel_count, n_sel: int, sel_size: int, shared: bool,
                    window: int, n_sink: int, cos_win, sin_win, seq_lens, out, ws: Optional[torch.Tensor] = None):
    """Attention over sinks, selection (tokens: sel_size 1, or blocks: sel_size cache.block) and window of a cache in 4 bits."""
    n_q = dims.batch * dims.n_q_heads * dims.head_dim
    n_h = dims.batch * (dims.n_kv_heads if shared else dims.n_q_heads)
    n_w = max(window, 1) * (dims.head_dim // 2)
    st = _cache_stream(dims, cache)
    rc = lib().a2ats_sparse_attn_kv4(ctypes.byref(dims), cache.ref, _arg(cache, q, "q", cache.kv_dtype, n_q),
                                     _arg(cache, q_rot, "q_rot", torch.float32, n_q),
                                     _arg(cache, sel_idx, "sel_idx", torch.int32, n_h * n_sel),
                                     _arg(cache, sel_count, "sel_count", torch.int32, n_h), n_sel, sel_size, int(shared), window,
                                     n_sink, _arg(cache, cos_win, "cos_win", torch.float32, n_w),
                                     _arg(cache, sin_win, "sin_win", torch.float32, n_w),
                                     _arg(cache, seq_lens, "seq_lens", torch.int32, dims.batch),
                                     _arg(cache, out, "out", cache.kv_dtype, n_q), _ws_ptr(cache, ws), _ws_bytes(ws), st)
    _check(rc, "a2ats_sparse_attn_kv4")


def _projected(dims: Dims, x: torch.Tensor, name: str, heads: int, n_new: int):
    """Pointer and token stride of [B, n_new, heads * D] (or [B, n_new, heads, D]) whose tokens are one distance apart."""
    B, D, s, four = dims.batch, dims.head_dim, x.stride(), x.dim() == 4
    if x.shape != ((B, n_new, heads, D) if four else (B, n_new, heads * D)):
        raise ValueError(f"{name} has shape {tuple(x.shape)}, not {(B, n_new, heads * D)}")
    # (the stride of an axis of length 1 says nothing)
    if s[-1] != 1 or (four and heads > 1 and s[2] != D):
        raise ValueError(f"{name}: the heads of a token lie behind each other")
    stride = s[1] if n_new > 1 else (s[0] if B > 1 else heads * D)
    if B > 1 and n_new > 0 and s[0] != n_new * stride:
        raise ValueError(f"{name}: all tokens are the same distance apart")
    return x.data_ptr(), stride


def qk_norm_rope(dims: Dims, q, k, n_new: int, q_weight, k_weight, eps: float, cos_pos, sin_pos, seq_lens=None, new_lens=None,
                 q_norm=None, k_norm=None, q_pos=None, k_pos=None):
    """Norms of the heads of q [B, n_new, Hq * D] and k [B, n_new, Hkv * D] (slices of one projection, or tensors of their own; either
    may be None), and their rotation by the tokens' positions (cos_pos, sin_pos [n_pos, D / 2], as rope_tables makes them for a
    window of n_pos >= ctx_len).  Outputs [B, H, n_new, D]: *_norm not rotated, *_pos rotated; those that are None are not made."""
    some = q if q is not None else k
    if some is None:
        raise ValueError("neither q nor k")
    dt, dev = some.dtype, some.get_device()
    if dev < 0:
        raise ValueError(f"the tensors are on {some.device}")
    if dev != torch.cuda.current_device():
        raise ValueError(f"the tensors are on {some.device}, the current device is {torch.cuda.current_device()}")
    code = _dtype_code(some)
    if q is not None and k is not None and (k.dtype is not dt or k.get_device() != dev):
        raise TypeError(f"k is {k.dtype} on {k.device}, not {dt} on {some.device}")
    B, D, Hq, Hkv = dims.batch, dims.head_dim, dims.n_q_heads, dims.n_kv_heads
    on = _Like(some, dev)
    n_pos = 0 if cos_pos is None else cos_pos.shape[0]
    n_q, n_k, n_cs, f32, i32 = B * Hq * n_new * D, B * Hkv * n_new * D, n_pos * (D // 2), torch.float32, torch.int32
    qp, qs = (None, 0) if q is None else _projected(dims, q, "q", Hq, n_new)
    kp, ks = (None, 0) if k is None else _projected(dims, k, "k", Hkv, n_new)
    rc = lib().a2ats_qk_norm_rope(ctypes.byref(dims), qp, qs, kp, ks, code, n_new,
                                  _arg(on, q_weight, "q_weight", f32, D), _arg(on, k_weight, "k_weight", f32, D),
                                  eps, _arg(on, cos_pos, "cos_pos", f32, n_cs), _arg(on, sin_pos, "sin_pos", f32, n_cs), n_pos,
                                  _arg(on, seq_lens, "seq_lens", i32, B), _arg(on, new_lens, "new_lens", i32, B),
                                  _arg(on, q_norm, "q_norm", dt, n_q), _arg(on, k_norm, "k_norm", dt, n_k),
                                  _arg(on, q_pos, "q_pos", dt, n_q), _arg(on, k_pos, "k_pos", dt, n_k),
                                  torch._C._cuda_getCurrentRawStream(dev))
    _check(rc, "a2ats_qk_norm_rope")


class _Like:
    """The device of a call's tensors, for _arg."""

    __slots__ = ("some", "device_index")

    def __init__(self, some, index):
        self.some, self.device_index = some, index

    @property
    def device(self):
        return self.some.device


def _ws_ptr(cache: KvBlocks, ws: Optional[torch.Tensor]):
    if ws is None:
        return None
    if ws.device != cache.device or not ws.is_contiguous():
        raise ValueError("the workspace is contiguous and on the cache's device")
    return ws.data_ptr()


def _ws_bytes(ws: Optional[torch.Tensor]) -> int:
    return 0 if ws is None else ws.numel() * ws.element_size()


PLAN_FIELDS = ("fast", "head_groups", "sample_parts", "sample_rows", "chunks", "rows_per_chunk",
               "segments_per_wave", "rows_per_segment", "segment_capacity", "survivor_capacity",
               "workspace_bytes_div_256")


def score_topk_plan(dims: Dims, top_k: int, window: int, n_sink: int) -> dict:
    """How a2ats_score_topk lays out its work for this shape (host only; no GPU needed)."""
    out = (ctypes.c_int32 * len(PLAN_FIELDS))()
    _check(lib().a2ats_score_topk_plan(ctypes.byref(dims), top_k, window, n_sink, out), "a2ats_score_topk_plan")
    return dict(zip(PLAN_FIELDS, (int(v) for v in out)))


def score_topk_stats(dims: Dims, top_k: int, window: int, n_sink: int, ws, cand_counts):
    rc = lib().a2ats_score_topk_stats(ctypes.byref(dims), top_k, window, n_sink, _ptr(ws), _ptr(cand_counts),
                                      _stream())
    _check(rc, "a2ats_score_topk_stats")


def score_topk_profiled(dims: Dims, codes, lut, lut_scale, top_k: int, window: int, n_sink: int, seq_lens,
                        topk_idx, topk_count, topk_score, scores_out, ws: Optional[torch.Tensor],
                        ev_start: int, ev_stop: int):
    """score_topk with a pair of HIP events (handles) attached to the dispatch of the code-streaming kernel."""
    rc = lib().a2ats_score_topk_profiled(ctypes.byref(dims), _ptr(codes), _ptr(lut), _ptr(lut_scale), top_k, window,
                                         n_sink, _ptr(seq_lens), _ptr(topk_idx), _ptr(topk_count), _ptr(topk_score),
                                         _ptr(scores_out), _ptr(ws),
                                         0 if ws is None else ws.numel() * ws.element_size(), _stream(),
                                         ctypes.c_void_p(ev_start), ctypes.c_void_p(ev_stop))
    _check(rc, "a2ats_score_topk_profiled")


class DecodeState:
    """Device buffers for one decode step of a fixed shape (allocation only; no arithmetic)."""

    def __init__(self, dims: Dims, top_k: int, window: int, n_sink: int, kv_dtype: torch.dtype,
                 inv_freq: torch.Tensor, wrope_b: int, device="cuda", want_scores=False):
        self.dims, self.top_k, self.window, self.n_sink = dims, top_k, window, n_sink
        B, Hq, D = dims.batch, dims.n_q_heads, dims.head_dim
        dev = torch.device(device)
        self.cos_b, self.sin_b, self.cos_win, self.sin_win = rope_tables(D, inv_freq, wrope_b, window, dev)
        self.q_rot = torch.empty(B, Hq, D, dtype=torch.float32, device=dev)
        self.lut = torch.empty(max(lut_elems(dims), 4), dtype=torch.int32, device=dev)
        self.lut_scale = torch.empty(B, Hq, dtype=torch.float32, device=dev)
        self.topk_idx = torch.empty(B, Hq, top_k, dtype=torch.int32, device=dev)
        self.topk_count = torch.empty(B, Hq, dtype=torch.int32, device=dev)
        self.topk_score = torch.empty(B, Hq, max(top_k, 1), dtype=torch.float32, device=dev)
        self.scores = torch.empty(B, Hq, dims.ctx_stride, dtype=torch.float32, device=dev) if want_scores else None
        self.out = torch.empty(B, Hq, D, dtype=kv_dtype, device=dev)
        n_ws = max(workspace_bytes(dims, OP_SCORE_TOPK, top_k, window),
                   workspace_bytes(dims, OP_ATTN, top_k, window),
                   workspace_bytes(dims, OP_ENCODE), 256)
        self.ws = torch.empty(n_ws, dtype=torch.uint8, device=dev)

    def step(self, q, codes, k_cache, v_cache, codebook, seq_lens=None, with_scores=False):
        """build_lut -> score_topk -> sparse_attn on the current stream; returns self.out."""
        build_lut(self.dims, q, self.cos_b, self.sin_b, codebook, self.q_rot, self.lut, self.lut_scale)
        score_topk(self.dims, codes, self.lut, self.lut_scale, self.top_k, self.window, self.n_sink, seq_lens,
                   self.topk_idx, self.topk_count, self.topk_score,
                   self.scores if with_scores else None, self.ws)
        sparse_attn(self.dims, q, self.q_rot, k_cache, v_cache, self.topk_idx, self.topk_count, self.top_k,
                    self.window, self.n_sink, self.cos_win, self.sin_win, seq_lens, self.out, self.ws)
        return self.out


class BlockDecodeState:
    """Device buffers for decode steps over a KvBlocks cache or a Kv4Cache with bounds (allocation only; no arithmetic).  scores:
    whether a step leaves the selected blocks' scores in block_score (which the attention does not need).  q_weight, k_weight, eps:
    of a model that normalises the heads of its queries and keys; a step then takes queries, keys and values as they come from the
    projections, slices of one tensor too (values that are one are copied first)."""

    def __init__(self, dims: Dims, cache, top_blocks: int, window: int, n_sink: int, inv_freq: torch.Tensor,
                 wrope_b: int, shared: bool = False, scores: bool = True, q_weight=None, k_weight=None, eps: float = 1e-6):
        self.dims, self.cache, self.top_blocks, self.window, self.n_sink, self.shared = dims, cache, top_blocks, window, n_sink, shared
        self.four_bits = isinstance(cache, Kv4Cache)
        self.blocks = cache.blocks if self.four_bits else cache
        if self.blocks is None or self.blocks.bounds is None:
            raise ValueError("blocks are selected by bounds, which the cache does not have")
        if (q_weight is None) != (k_weight is None):
            raise ValueError("q_weight and k_weight are given together")
        self.q_weight, self.k_weight, self.eps = q_weight, k_weight, eps
        B, Hq, Hkv, D, dev = dims.batch, dims.n_q_heads, dims.n_kv_heads, dims.head_dim, cache.device
        heads = Hkv if shared else Hq
        self.cos_b, self.sin_b, self.cos_win, self.sin_win = rope_tables(D, inv_freq, wrope_b, window, dev)
        self.q_rot = torch.empty(B, Hq, D, dtype=torch.float32, device=dev)
        self.block_idx = torch.empty(B, heads, top_blocks, dtype=torch.int32, device=dev)
        self.block_count = torch.empty(B, heads, dtype=torch.int32, device=dev)
        self.block_score = torch.empty(B, heads, top_blocks, dtype=torch.float32, device=dev) if scores else None
        self.out = torch.empty(B, Hq, D, dtype=cache.kv_dtype, device=dev)
        if q_weight is not None:
            self.q_norm = torch.empty(B, Hq, D, dtype=cache.kv_dtype, device=dev)
            self.k_norm = torch.empty(B, Hkv, 1, D, dtype=cache.kv_dtype, device=dev)
            self.v_new = torch.empty(B, Hkv, 1, D, dtype=cache.kv_dtype, device=dev)
        n_ws = max(workspace_bytes(dims, OP_BLOCK_TOPK),
                   workspace_bytes(dims, OP_ATTN_KV4 if self.four_bits else OP_ATTN_KV8, top_blocks * cache.block, window), 256)
        self.ws = torch.empty(n_ws, dtype=torch.uint8, device=dev)

    def step(self, q, k_new, v_new, seq_lens=None):
        """qk_norm_rope (if there are weights) -> append of one token a sequence -> block_topk -> attention on the current stream;
        returns self.out.  q [B, Hq, D], k_new, v_new [B, Hkv, 1, D].
        seq_lens counts that token already and is at most dims.ctx_len (None: ctx_len): a cache is made with room for what it
        is to hold, a larger length is taken as ctx_len and the token replaces the last one."""
        dims = self.dims
        append, attend = (kv4_append, sparse_attn_kv4) if self.four_bits else (kv8_append, sparse_attn_kv8)
        if self.q_weight is not None:
            qk_norm_rope(dims, q.reshape(dims.batch, 1, -1), k_new.reshape(dims.batch, 1, -1), 1, self.q_weight, self.k_weight, self.eps,
                         None, None, seq_lens, None, q_norm=self.q_norm, k_norm=self.k_norm)
            q, k_new = self.q_norm, self.k_norm
            if not v_new.is_contiguous() and v_new.shape == self.v_new.shape and v_new.dtype == self.v_new.dtype and v_new.device == self.v_new.device:
                v_new = self.v_new.copy_(v_new)            # (what does not fit is the append's to refuse)
        append(dims, self.cache, k_new, v_new, 1, seq_lens)
        block_topk(dims, self.blocks, q, self.cos_b, self.sin_b, self.q_rot, self.shared, self.top_blocks, self.window,
                   self.n_sink, seq_lens, self.block_idx, self.block_count, self.block_score, ws=self.ws)
        attend(dims, self.cache, q, self.q_rot, self.block_idx, self.block_count, self.top_blocks, self.cache.block,
               self.shared, self.window, self.n_sink, self.cos_win, self.sin_win, seq_lens, self.out, self.ws)
        return self.out
