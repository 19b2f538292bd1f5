"""ctypes binding of libadadsf.so: the C ABI in include/adadsf.h, one Python
function per entry point, same names without the ``dsf_`` prefix.

Argument marshalling only. Tensors are torch tensors on the GPU (torch owns
device memory and streams); every computation runs in the library's HIP
kernels. A missing library raises immediately: there is no fallback path.
"""
from __future__ import annotations

import contextlib
import ctypes
import os
from typing import Optional, Sequence

import torch  # loads the HIP runtime that the library binds to

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libadadsf.so")

F32, BF16 = 0, 1
E4M3 = 2  # elements of a paged cache only
PAGE_SIZES = (16, 32, 64, 128, 256)
BLOCK_NEOX_PARALLEL, BLOCK_QWEN_SEQ = 0, 1
FLAG_DENSE, FLAG_GATE = 1, 2
CLIP = {"none": 0, "plain": 1, "budget": 2}
ROUNDING = {"floor": 0, "ceil": 1}
KINDS = ["sim", "router", "topk", "norm", "gemm_qkv", "attn", "gemm_o", "gemm_up", "gemm_down",
         "gather", "scatter", "other", "backward", "align"]

STATUS = {0: "DSF_OK", 1: "DSF_EINVAL", 2: "DSF_EUNSUPPORTED", 3: "DSF_EWORKSPACE", 4: "DSF_EHIP",
          5: "DSF_ENODEVICE"}

EXPORTS = [
    "dsf_version", "dsf_last_error", "dsf_sim_workspace_size", "dsf_sim_stats", "dsf_sim_finalize",
    "dsf_retention_from_similarity", "dsf_k_from_retention", "dsf_router_score", "dsf_topk_select",
    "dsf_gather_rows", "dsf_scatter_residual", "dsf_attention_forward", "dsf_workspace_size",
    "dsf_sparse_block_forward", "dsf_stack_forward", "dsf_timing_enable", "dsf_timing_read",
    "dsf_gate_score_grad", "dsf_router_backward_workspace_size", "dsf_router_backward",
    "dsf_align_workspace_size", "dsf_align_hidden", "dsf_kl_align", "dsf_align_stack_workspace_size",
    "dsf_align_stack_forward", "dsf_decode_workspace_size", "dsf_decode_step", "dsf_stack_prefill",
    "dsf_workspace_status", "dsf_decode_static_scratch_bytes", "dsf_decode_step_static",
    "dsf_backward_workspace_size", "dsf_sparse_block_backward",
    "dsf_paged_cache_write", "dsf_paged_cache_read", "dsf_paged_attention_workspace_size", "dsf_paged_attention",
    "dsf_embed_forward", "dsf_embed_backward_workspace_size", "dsf_embed_backward", "dsf_norm_forward",
    "dsf_norm_backward_workspace_size", "dsf_norm_backward", "dsf_head_workspace_size", "dsf_head_cross_entropy",
    "dsf_head_distill",
]
WS_STATUS_SK_TIMEOUT = 1


class DsfError(RuntimeError):
    def __init__(self, fn: str, code: int, msg: str):
        super().__init__(f"{fn} -> {STATUS.get(code, code)}: {msg}")
        self.code = code


class LayerDesc(ctypes.Structure):
    _fields_ = [("block", ctypes.c_int32), ("d_model", ctypes.c_int32), ("n_heads", ctypes.c_int32),
                ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("d_ff", ctypes.c_int32),
                ("rotary_dims", ctypes.c_int32), ("d_router", ctypes.c_int32), ("norm_eps", ctypes.c_float),
                ("reserved", ctypes.c_float), ("rope_theta", ctypes.c_double)]


_WEIGHT_FIELDS = ["router_w1", "router_b1", "router_w2", "router_b2", "reserved", "norm1_w", "norm1_b",
                  "norm2_w", "norm2_b", "w_qkv", "b_qkv", "w_o", "b_o", "w_up", "b_up", "w_down", "b_down"]


GRAD_FIELDS = ["w_qkv", "b_qkv", "w_o", "b_o", "w_up", "b_up", "w_down", "b_down", "norm1_w", "norm1_b",
               "norm2_w", "norm2_b"]


class LayerGrads(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in GRAD_FIELDS]


class _PagedCacheStruct(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("k", "v", "k_exp", "v_exp")] + \
        [(n, ctypes.c_int32) for n in ("type", "n_pages", "n_kv_heads", "page_size", "head_dim", "reserved")]


class _PagedBatchStruct(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("row_start", "kv_len", "pages")] + \
        [(n, ctypes.c_int32) for n in ("B", "max_pages", "n_rows", "max_rows")]


class LayerWeights(ctypes.Structure):
    _fields_ = [(n, ctypes.c_float if n in ("router_b2", "reserved") else ctypes.c_void_p)
                for n in _WEIGHT_FIELDS]


_lib = None


def lib() -> ctypes.CDLL:
    """The loaded library; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with __graft_entry__.build() "
                           "(python -m paper_2607_21291_amd.build_lib)")
    L = ctypes.CDLL(LIB_PATH)
    vp, i32, i64, sz, f32, f64 = (ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_size_t,
                                  ctypes.c_float, ctypes.c_double)
    sig = {
        "dsf_version": ([], i32),
        "dsf_last_error": ([], ctypes.c_char_p),
        "dsf_sim_workspace_size": ([i64], sz),
        "dsf_sim_stats": ([vp, vp, i32, i64, i32, vp, vp, vp, sz, vp], i32),
        "dsf_sim_finalize": ([vp, i32, vp, vp], i32),
        "dsf_retention_from_similarity": ([vp, i32, f64, f64, f64, i32, vp], i32),
        "dsf_k_from_retention": ([f64, i32, i32], i32),
        "dsf_router_score": ([vp, i32, i64, i32, i32, vp, vp, vp, f32, vp, vp], i32),
        "dsf_topk_select": ([vp, i32, i32, i32, vp, vp], i32),
        "dsf_gather_rows": ([vp, i32, i32, i32, i32, vp, i32, vp, vp], i32),
        "dsf_scatter_residual": ([vp, vp, i32, i32, i32, i32, vp, i32, vp], i32),
        "dsf_attention_forward": ([vp, vp, vp, i32, i32, i32, i32, i32, i32, vp, vp], i32),
        "dsf_workspace_size": ([vp, i32, i32, i32, i32, i32], sz),
        "dsf_workspace_status": ([vp, vp, vp], i32),
        "dsf_sparse_block_forward": ([vp, vp, i32, vp, i32, i32, i32, i32, vp, vp, vp, vp, sz, vp], i32),
        "dsf_stack_forward": ([vp, vp, i32, i32, vp, vp, i32, i32, i32, vp, vp, sz, vp], i32),
        "dsf_timing_enable": ([i32, ctypes.c_uint32], i32),
        "dsf_timing_read": ([i32, vp, vp], i32),
        "dsf_gate_score_grad": ([vp, vp, vp, i32, vp, vp, i32, i32, i32, i32, vp, vp], i32),
        "dsf_router_backward_workspace_size": ([i64, i32, i32], sz),
        "dsf_router_backward": ([vp, i32, i64, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp], i32),
        "dsf_align_workspace_size": ([i64], sz),
        "dsf_align_hidden": ([vp, vp, i32, i64, i32, vp, vp, vp, sz, vp], i32),
        "dsf_kl_align": ([vp, vp, i32, i64, i32, vp, vp, vp, sz, vp], i32),
        "dsf_align_stack_workspace_size": ([vp, i32, i32, i32], sz),
        "dsf_align_stack_forward": ([vp, vp, i32, i32, vp, vp, vp, i32, i32, i32, vp, vp, sz, vp], i32),
        "dsf_decode_workspace_size": ([vp, i32, i32, i32, i32], sz),
        "dsf_decode_step": ([vp, vp, i32, i32, vp, i32, vp, i32, vp, vp, vp, vp, vp, vp, i32, vp, sz, vp], i32),
        "dsf_stack_prefill": ([vp, vp, i32, i32, vp, vp, i32, i32, vp, vp, vp, i32, vp, vp, sz, vp], i32),
        "dsf_decode_static_scratch_bytes": ([], sz),
        "dsf_backward_workspace_size": ([vp, i32, i32, i32, i32], sz),
        "dsf_sparse_block_backward": ([vp, vp, i32, vp, vp, i32, i32, i32, vp, vp, i32, vp, vp, vp, sz, vp], i32),
        "dsf_decode_step_static": ([vp, vp, i32, i32, vp, i32, vp, i32, vp, vp, vp, vp, vp, vp, i32, vp], i32),
        "dsf_paged_cache_write": ([vp, vp, i32, vp, i64, i64, vp, i64, i64, vp], i32),
        "dsf_paged_cache_read": ([vp, vp, i32, vp, i64, i64, vp, i64, i64, vp], i32),
        "dsf_paged_attention_workspace_size": ([vp, vp, i32, i32], sz),
        "dsf_paged_attention": ([vp, vp, i32, i32, vp, i64, i64, i32, vp, i64, i64, vp, sz, vp], i32),
        "dsf_embed_forward": ([vp, vp, i32, i64, i32, i32, f32, vp, vp], i32),
        "dsf_embed_backward_workspace_size": ([i64, i32, i32], sz),
        "dsf_embed_backward": ([vp, vp, i32, i64, i32, i32, f32, i32, vp, i32, vp, sz, vp], i32),
        "dsf_norm_forward": ([vp, vp, vp, i32, i64, i32, f32, i32, vp, vp], i32),
        "dsf_norm_backward_workspace_size": ([i64, i32], sz),
        "dsf_norm_backward": ([vp, vp, vp, vp, i32, i64, i32, f32, i32, vp, vp, vp, vp, sz, vp], i32),
        "dsf_head_workspace_size": ([i32, i64, i32, i32, i32, i32], sz),
        "dsf_head_cross_entropy": ([vp, vp, i32, i64, i32, i32, vp, vp, f32, i32, vp, vp, vp, vp, i32, vp, sz, vp], i32),
        "dsf_head_distill": ([vp, vp, i32, i64, i32, i32, vp, vp, i32, f32, vp, f32, i32, vp, vp, vp, vp, i32, vp, sz, vp],
                             i32),
    }
    for name, (args, res) in sig.items():
        fn = getattr(L, name)
        fn.argtypes = args
        fn.restype = res
    _lib = L
    return L


def _check(fn: str, rc: int):
    if rc != 0:
        raise DsfError(fn, rc, lib().dsf_last_error().decode())


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    if not t.is_contiguous():
        raise ValueError("tensors passed to the library must be contiguous")
    return t.data_ptr()


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise ValueError(f"unsupported dtype {t.dtype}")


# the current stream's handle without building a Stream object (1.5 us of a
# 6 us call); the public accessor where this build of torch lacks it
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream) -> int:
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


# --------------------------------------------------------------- entry points

def version() -> int:
    return lib().dsf_version()


def last_error() -> str:
    return lib().dsf_last_error().decode()


def sim_workspace_size(n_tokens: int) -> int:
    return lib().dsf_sim_workspace_size(n_tokens)


def sim_stats(x_in, x_out, accum, per_token_cos=None, workspace=None, stream=None):
    d = x_in.shape[-1]
    n = x_in.numel() // d
    if workspace is None:
        workspace = torch.empty(max(sim_workspace_size(n), 256), dtype=torch.uint8, device=x_in.device)
    _check("dsf_sim_stats", lib().dsf_sim_stats(_ptr(x_in), _ptr(x_out), _dtype_code(x_in), n, d,
                                                _ptr(per_token_cos), _ptr(accum), _ptr(workspace),
                                                workspace.numel(), _stream(stream)))


def sim_finalize(accum, stream=None):
    L = accum.numel() // 2
    out = (ctypes.c_double * max(L, 1))()
    _check("dsf_sim_finalize", lib().dsf_sim_finalize(_ptr(accum), L, ctypes.addressof(out), _stream(stream)))
    return [out[i] for i in range(L)]


def retention_from_similarity(s: Sequence[float], t: float, tau: Optional[float], beta: float = 10.0,
                              clip: str = "budget"):
    L = len(s)
    sin = (ctypes.c_double * max(L, 1))(*s)
    rout = (ctypes.c_double * max(L, 1))()
    _check("dsf_retention_from_similarity",
           lib().dsf_retention_from_similarity(ctypes.addressof(sin), L, t, -1.0 if tau is None else tau, beta,
                                               CLIP[clip], ctypes.addressof(rout)))
    return [rout[i] for i in range(L)]


def k_from_retention(r: float, T: int, rounding: str = "floor") -> int:
    k = lib().dsf_k_from_retention(r, T, ROUNDING[rounding])
    if k < 0:
        raise DsfError("dsf_k_from_retention", 1, last_error())
    return k


def router_score(x, w1, b1, w2, b2: float, scores, stream=None):
    d = x.shape[-1]
    _check("dsf_router_score", lib().dsf_router_score(_ptr(x), _dtype_code(x), x.numel() // d, d, w1.shape[0],
                                                      _ptr(w1), _ptr(b1), _ptr(w2), float(b2), _ptr(scores),
                                                      _stream(stream)))


def gate_score_grad(dy, x_in, x_out, scores, idx, dscore, stream=None):
    B, T, d = dy.shape
    _check("dsf_gate_score_grad",
           lib().dsf_gate_score_grad(_ptr(dy), _ptr(x_in), _ptr(x_out), _dtype_code(dy), _ptr(scores), _ptr(idx),
                                     B, T, idx.shape[1], d, _ptr(dscore), _stream(stream)))


def router_backward_workspace_size(n_tokens: int, d: int, d_r: int) -> int:
    return lib().dsf_router_backward_workspace_size(n_tokens, d, d_r)


def router_backward(x, w1, b1, w2, dscore, dw1, db1, dw2, db2, dx=None, workspace=None, stream=None):
    d = x.shape[-1]
    n = x.numel() // d
    d_r = w1.shape[0]
    if workspace is None:
        workspace = torch.empty(max(router_backward_workspace_size(n, d, d_r), 256), dtype=torch.uint8,
                                device=x.device)
    _check("dsf_router_backward",
           lib().dsf_router_backward(_ptr(x), _dtype_code(x), n, d, d_r, _ptr(w1), _ptr(b1), _ptr(w2), _ptr(dscore),
                                     _ptr(dw1), _ptr(db1), _ptr(dw2), _ptr(db2), _ptr(dx), _ptr(workspace),
                                     workspace.numel(), _stream(stream)))


def topk_select(scores, k: int, idx, stream=None):
    B, T = scores.shape
    _check("dsf_topk_select", lib().dsf_topk_select(_ptr(scores), B, T, k, _ptr(idx), _stream(stream)))


def gather_rows(x, idx, out, stream=None):
    B, T, d = x.shape
    _check("dsf_gather_rows", lib().dsf_gather_rows(_ptr(x), _dtype_code(x), B, T, d, _ptr(idx), idx.shape[1],
                                                    _ptr(out), _stream(stream)))


def scatter_residual(x, delta, idx, stream=None):
    B, T, d = x.shape
    _check("dsf_scatter_residual", lib().dsf_scatter_residual(_ptr(x), _ptr(delta), _dtype_code(x), B, T, d,
                                                              _ptr(idx), idx.shape[1], _stream(stream)))


def attention_forward(q, k, v, out, stream=None):
    B, Hq, n, hd = q.shape
    _check("dsf_attention_forward", lib().dsf_attention_forward(_ptr(q), _ptr(k), _ptr(v), _dtype_code(q), B, Hq,
                                                                k.shape[1], n, hd, _ptr(out), _stream(stream)))


def workspace_size(desc: LayerDesc, dtype: int, B: int, T: int, k_max: int, with_similarity: bool = False) -> int:
    return lib().dsf_workspace_size(ctypes.addressof(desc), dtype, B, T, k_max, int(with_similarity))


def workspace_status(workspace, stream=None) -> int:
    """Status word of the last layer/stack call on this workspace (waits for the stream)."""
    out = ctypes.c_uint32(0)
    _check("dsf_workspace_status", lib().dsf_workspace_status(_ptr(workspace), ctypes.byref(out), _stream(stream)))
    return int(out.value)


def backward_workspace_size(desc: LayerDesc, dtype: int, B: int, T: int, k: int) -> int:
    return lib().dsf_backward_workspace_size(ctypes.addressof(desc), dtype, B, T, k)


def sparse_block_backward(desc: LayerDesc, weights: LayerWeights, x, dy, idx, dx, grads: dict, workspace,
                          scores=None, flags: int = 0, stream=None):
    """grads: name -> fp32 device tensor (or None) for the names in GRAD_FIELDS."""
    B, T, _ = x.shape
    k = idx.shape[1] if idx is not None else 0
    gs = LayerGrads(*[_ptr(grads.get(n)) for n in GRAD_FIELDS])
    _check("dsf_sparse_block_backward",
           lib().dsf_sparse_block_backward(ctypes.addressof(desc), ctypes.addressof(weights), _dtype_code(x),
                                           _ptr(x), _ptr(dy), B, T, k, _ptr(idx), _ptr(scores), flags, _ptr(dx),
                                           ctypes.addressof(gs), _ptr(workspace), workspace.numel(),
                                           _stream(stream)))


def sparse_block_forward(desc: LayerDesc, weights: LayerWeights, x, k: int, workspace, flags: int = 0,
                         scores_out=None, idx_out=None, idx_in=None, stream=None):
    B, T, _ = x.shape
    _check("dsf_sparse_block_forward",
           lib().dsf_sparse_block_forward(ctypes.addressof(desc), ctypes.addressof(weights), _dtype_code(x),
                                          _ptr(x), B, T, k, flags, _ptr(scores_out), _ptr(idx_out), _ptr(idx_in),
                                          _ptr(workspace), workspace.numel(), _stream(stream)))


def stack_forward(desc: LayerDesc, weights: Sequence[LayerWeights], ks: Sequence[int], x, workspace,
                  flags: int = 0, sim_accum=None, stream=None):
    B, T, _ = x.shape
    L = len(weights)
    arr = (LayerWeights * max(L, 1))(*weights)
    karr = (ctypes.c_int * max(L, 1))(*[int(k) for k in ks])
    _check("dsf_stack_forward",
           lib().dsf_stack_forward(ctypes.addressof(desc), ctypes.addressof(arr), L, _dtype_code(x),
                                   ctypes.addressof(karr), _ptr(x), B, T, flags, _ptr(sim_accum), _ptr(workspace),
                                   workspace.numel(), _stream(stream)))


def align_workspace_size(n_rows: int) -> int:
    return lib().dsf_align_workspace_size(n_rows)


def align_hidden(h_sparse, h_dense, accum, per_token_sq=None, workspace=None, stream=None):
    d = h_sparse.shape[-1]
    n = h_sparse.numel() // d
    if workspace is None:
        workspace = torch.empty(align_workspace_size(n), dtype=torch.uint8, device=h_sparse.device)
    _check("dsf_align_hidden", lib().dsf_align_hidden(_ptr(h_sparse), _ptr(h_dense), _dtype_code(h_sparse), n, d,
                                                      _ptr(per_token_sq), _ptr(accum), _ptr(workspace),
                                                      workspace.numel(), _stream(stream)))


def kl_align(logits_dense, logits_sparse, accum, per_row_kl=None, workspace=None, stream=None):
    C = logits_dense.shape[-1]
    n = logits_dense.numel() // C
    if workspace is None:
        workspace = torch.empty(align_workspace_size(n), dtype=torch.uint8, device=logits_dense.device)
    _check("dsf_kl_align", lib().dsf_kl_align(_ptr(logits_dense), _ptr(logits_sparse), _dtype_code(logits_dense), n,
                                              C, _ptr(per_row_kl), _ptr(accum), _ptr(workspace), workspace.numel(),
                                              _stream(stream)))


def align_stack_workspace_size(desc: LayerDesc, dtype: int, B: int, T: int) -> int:
    return lib().dsf_align_stack_workspace_size(ctypes.addressof(desc), dtype, B, T)


def align_stack_forward(desc: LayerDesc, weights: Sequence[LayerWeights], ks: Sequence[int], x_sparse, x_dense,
                        hid_accum, workspace, flags: int = 0, stream=None):
    B, T, _ = x_sparse.shape
    L = len(weights)
    arr = (LayerWeights * max(L, 1))(*weights)
    karr = (ctypes.c_int * max(L, 1))(*[int(k) for k in ks])
    _check("dsf_align_stack_forward",
           lib().dsf_align_stack_forward(ctypes.addressof(desc), ctypes.addressof(arr), L, _dtype_code(x_sparse),
                                         ctypes.addressof(karr), _ptr(x_sparse), _ptr(x_dense), B, T, flags,
                                         _ptr(hid_accum), _ptr(workspace), workspace.numel(), _stream(stream)))


def decode_workspace_size(desc: LayerDesc, dtype: int, B: int, max_pos: int, cap: int) -> int:
    return lib().dsf_decode_workspace_size(ctypes.addressof(desc), dtype, B, max_pos, cap)


def _ptr_array(tensors):
    return (ctypes.c_void_p * max(len(tensors), 1))(*[_ptr(t) for t in tensors])


def decode_step(desc: LayerDesc, weights: Sequence[LayerWeights], x, pos, max_pos: int, thr, cache_k, cache_v,
                cache_len, workspace, scores_out=None, keep_out=None, stream=None):
    """x [B, d]; pos int32 [B]; thr float [L, B]; cache_k / cache_v: L tensors [B, Hkv, cap, hd];
    cache_len int32 [L, B]."""
    B = x.shape[0]
    L = len(weights)
    cap = cache_k[0].shape[2] if L else 1
    arr = (LayerWeights * max(L, 1))(*weights)
    ck, cv = _ptr_array(cache_k), _ptr_array(cache_v)
    _check("dsf_decode_step",
           lib().dsf_decode_step(ctypes.addressof(desc), ctypes.addressof(arr), L, _dtype_code(x), _ptr(x), B,
                                 _ptr(pos), max_pos, _ptr(thr), _ptr(scores_out), _ptr(keep_out),
                                 ctypes.addressof(ck), ctypes.addressof(cv), _ptr(cache_len), cap, _ptr(workspace),
                                 workspace.numel(), _stream(stream)))


def decode_static_scratch_bytes() -> int:
    return lib().dsf_decode_static_scratch_bytes()


def decode_step_static(desc: LayerDesc, weights: Sequence[LayerWeights], x, pos, max_pos: int, thr, cache_k,
                       cache_v, cache_len, scores_out=None, keep_out=None, stream=None):
    """dsf_decode_step on the library's static device scratch (no workspace, no allocation)."""
    B = x.shape[0]
    L = len(weights)
    cap = cache_k[0].shape[2] if L else 1
    arr = (LayerWeights * max(L, 1))(*weights)
    ck, cv = _ptr_array(cache_k), _ptr_array(cache_v)
    _check("dsf_decode_step_static",
           lib().dsf_decode_step_static(ctypes.addressof(desc), ctypes.addressof(arr), L, _dtype_code(x), _ptr(x), B,
                                        _ptr(pos), max_pos, _ptr(thr), _ptr(scores_out), _ptr(keep_out),
                                        ctypes.addressof(ck), ctypes.addressof(cv), _ptr(cache_len), cap,
                                        _stream(stream)))


def stack_prefill(desc: LayerDesc, weights: Sequence[LayerWeights], ks: Sequence[int], x, cache_k, cache_v,
                  cache_len, workspace, thr_out=None, stream=None):
    """dsf_stack_forward over x [B, T, d] that also fills the decode caches."""
    B, T, _ = x.shape
    L = len(weights)
    cap = cache_k[0].shape[2] if L else 1
    arr = (LayerWeights * max(L, 1))(*weights)
    karr = (ctypes.c_int * max(L, 1))(*[int(k) for k in ks])
    ck, cv = _ptr_array(cache_k), _ptr_array(cache_v)
    _check("dsf_stack_prefill",
           lib().dsf_stack_prefill(ctypes.addressof(desc), ctypes.addressof(arr), L, _dtype_code(x),
                                   ctypes.addressof(karr), _ptr(x), B, T, ctypes.addressof(ck), ctypes.addressof(cv),
                                   _ptr(cache_len), cap, _ptr(thr_out), _ptr(workspace), workspace.numel(),
                                   _stream(stream)))


class PagedCache:
    """Pages of one layer's keys and values: k, v [n_pages, n_kv_heads, page_size, head_dim] of torch.float32,
    torch.bfloat16 or torch.float8_e4m3fn codes, these with k_exp, v_exp uint8 [n_pages, n_kv_heads, page_size]
    (a code counts 2^(byte - 127)). Keeps the tensors; the calls take it wherever they take a cache."""

    def __init__(self, k, v, k_exp=None, v_exp=None):
        types = {torch.float32: F32, torch.bfloat16: BF16, torch.float8_e4m3fn: E4M3}
        if k.dim() != 4 or v.shape != k.shape or v.dtype != k.dtype or k.dtype not in types:
            raise ValueError("k and v: [n_pages, n_kv_heads, page_size, head_dim], both float32, bfloat16 or float8_e4m3fn")
        codes = types[k.dtype] == E4M3
        for t in (k_exp, v_exp):
            if (t is not None) != codes or (codes and (t.dtype != torch.uint8 or t.shape != k.shape[:3])):
                raise ValueError("k_exp and v_exp: uint8 [n_pages, n_kv_heads, page_size] for float8_e4m3fn pages, "
                                 "None for others")
        self.k, self.v, self.k_exp, self.v_exp = k, v, k_exp, v_exp
        self.device = _one_device(*(t for t in (k, v, k_exp, v_exp) if t is not None))
        self.index = k.get_device()  # -1: not on a GPU
        n_pages, heads, page, hd = k.shape
        self.n_kv_heads, self.head_dim = heads, hd
        self._struct = _PagedCacheStruct(_ptr(k), _ptr(v), _ptr(k_exp), _ptr(v_exp), types[k.dtype], n_pages, heads, page,
                                         hd, 0)
        self._addr = ctypes.addressof(self._struct)

    @classmethod
    def empty(cls, n_pages: int, n_kv_heads: int, page_size: int, head_dim: int, dtype, device):
        """A pool of uninitialised pages (no slot is read before it is written)."""
        shape = (n_pages, n_kv_heads, page_size, head_dim)
        k, v = (torch.empty(shape, dtype=dtype, device=device) for _ in range(2))
        exps = [None, None]
        if dtype == torch.float8_e4m3fn:
            exps = [torch.empty(shape[:3], dtype=torch.uint8, device=device) for _ in range(2)]
        return cls(k, v, *exps)


class PagedBatch:
    """One step's sequences on paged caches: row_start int32 [B + 1], kv_len int32 [B], pages int32 [B, max_pages]
    on the device, for tensors of n_rows rows; max_rows: at least every sequence's rows. Keeps the tensors, whose
    values may change between calls (also between replays of a captured one)."""

    def __init__(self, row_start, kv_len, pages, n_rows: int, max_rows: int):
        if any(t.dtype != torch.int32 for t in (row_start, kv_len, pages)):
            raise ValueError("row_start, kv_len and pages must be int32")
        B = kv_len.shape[0] if kv_len.dim() == 1 else -1
        if B < 0 or row_start.shape != (B + 1,) or pages.dim() != 2 or pages.shape[0] != B:
            raise ValueError("row_start [B + 1], kv_len [B], pages [B, max_pages]")
        if not (0 <= n_rows < 2**31 and 0 <= max_rows < 2**31):
            raise ValueError("n_rows and max_rows must be from 0 to 2^31 - 1")
        self.row_start, self.kv_len, self.pages, self.n_rows = row_start, kv_len, pages, n_rows
        self.device = _one_device(row_start, kv_len, pages)
        self.index = kv_len.get_device()
        self._struct = _PagedBatchStruct(_ptr(row_start), _ptr(kv_len), _ptr(pages), B, pages.shape[1], n_rows, max_rows)
        self._addr = ctypes.addressof(self._struct)


def _one_device(*tensors):
    device = tensors[0].device
    if any(t.device != device for t in tensors):
        raise ValueError("the tensors lie on different devices")
    return device


def _paged_rows(name: str, t, cache: PagedCache, batch: PagedBatch, heads: Optional[int] = None):
    """Pointer and strides of rows [n_rows, heads, head_dim] (last dimension contiguous)."""
    shape = t.shape
    if len(shape) != 3 or shape[0] != batch.n_rows or shape[2] != cache.head_dim or (heads is not None and shape[1] != heads):
        raise ValueError(f"{name}: [n_rows, heads, head_dim] = [{batch.n_rows}, {heads or 'heads'}, {cache.head_dim}] "
                         f"expected, got {list(shape)}")
    if t.get_device() != cache.index:
        raise ValueError(f"{name} lies on {t.device}, the cache on {cache.device}")
    row, head, last = t.stride()
    if last != 1:
        raise ValueError(f"{name}: the last dimension must be contiguous")
    # strides of dimensions of size one say nothing
    return t.data_ptr(), row if shape[0] > 1 else 0, head if shape[1] > 1 else 0


def _paged_call(name: str, cache: PagedCache, batch: PagedBatch, stream, *args):
    """The C entry point `name` with the caches' device current, on the given stream or that device's current one."""
    index = cache.index
    if index < 0:
        raise ValueError(f"the tensors lie on {cache.device}, not on a GPU")
    if batch.index != index:
        raise ValueError(f"the batch lies on {batch.device}, the cache on {cache.device}")
    if stream is not None and stream.device.index != index:
        raise ValueError(f"the stream belongs to {stream.device}, the tensors to {cache.device}")
    fn = getattr(_lib or lib(), name)
    if index == torch.cuda.current_device():
        rc = fn(cache._addr, batch._addr, *args, _stream(stream))
    else:
        with torch.cuda.device(index):
            rc = fn(cache._addr, batch._addr, *args, _stream(stream))
    if rc:
        _check(name, rc)


def paged_cache_write(cache: PagedCache, batch: PagedBatch, k, v, stream=None):
    """k, v [n_rows, n_kv_heads, head_dim] (views of wider rows, too) into the slots of the batch's rows."""
    heads = cache.n_kv_heads
    if v.dtype != k.dtype:
        raise ValueError("k and v have different dtypes")
    _paged_call("dsf_paged_cache_write", cache, batch, stream, _dtype_code(k), *_paged_rows("k", k, cache, batch, heads),
                *_paged_rows("v", v, cache, batch, heads))


def paged_cache_read(cache: PagedCache, batch: PagedBatch, k, v, stream=None):
    """The slots of the batch's rows into k, v [n_rows, n_kv_heads, head_dim]; other rows stay as they are."""
    heads = cache.n_kv_heads
    if v.dtype != k.dtype:
        raise ValueError("k and v have different dtypes")
    _paged_call("dsf_paged_cache_read", cache, batch, stream, _dtype_code(k), *_paged_rows("k", k, cache, batch, heads),
                *_paged_rows("v", v, cache, batch, heads))


def paged_attention_workspace_size(cache: PagedCache, batch: PagedBatch, dtype: int, n_heads: int) -> int:
    return lib().dsf_paged_attention_workspace_size(cache._addr, batch._addr, dtype, n_heads)


def paged_attention(cache: PagedCache, batch: PagedBatch, q, out, window: int = 0, workspace=None, stream=None):
    """q [n_rows, n_heads, head_dim] over the pages; out the same shape. Rows of no sequence stay as they are."""
    qp, heads = _paged_rows("q", q, cache, batch), q.shape[1]
    op = _paged_rows("out", out, cache, batch, heads)
    if out.dtype != q.dtype:
        raise ValueError("q and out have different dtypes")
    if not 0 <= window < 2**31:
        raise ValueError("window must be from 0 to 2^31 - 1")
    dtype = _dtype_code(q)
    if workspace is None:
        need = max(paged_attention_workspace_size(cache, batch, dtype, heads), 256)
        # on the stream that uses it, so that its memory is not handed on before that
        with torch.cuda.stream(stream) if stream is not None else contextlib.nullcontext():
            workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
    elif workspace.get_device() != cache.index:
        raise ValueError(f"workspace lies on {workspace.device}, the cache on {cache.device}")
    elif not workspace.is_contiguous():
        raise ValueError("the workspace must be contiguous")
    _paged_call("dsf_paged_attention", cache, batch, stream, dtype, heads, *qp, window, *op, workspace.data_ptr(),
                workspace.nbytes)


# ------------------------------------- the ends of a training step: embedding, norm, head

def _dense(name: str, t, shape, dtype, index, other=None):
    """Pointer of a contiguous tensor of that shape, of dtype (or `other`), on device `index` (None: null)."""
    if t is None:
        return None
    if t.dtype is dtype and t.is_contiguous() and t.get_device() == index and t.shape == shape:
        return t.data_ptr()
    if t.dtype not in (dtype, other):
        raise ValueError(f"{name}: {dtype}{f' or {other}' if other else ''} expected, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name}: shape {list(shape)} expected, got {list(t.shape)}")
    if t.get_device() != index:
        raise ValueError(f"{name} lies on {t.device}, the call's other tensors do not")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _scratch(workspace, size, like, stream):
    """Pointer, bytes and the tensor of a call's workspace: the caller's, or a new one of size() bytes."""
    if workspace is None:
        need = size()
        # on the stream that uses it, so that its memory is not handed on before that
        with torch.cuda.stream(stream) if stream is not None else contextlib.nullcontext():
            workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=like.device)
    elif workspace.get_device() != like.get_device():
        raise ValueError(f"workspace lies on {workspace.device}, not on {like.device}")
    elif not workspace.is_contiguous():
        raise ValueError("the workspace must be contiguous")
    return workspace.data_ptr(), workspace.nbytes, workspace


def _call_on(name: str, like, index: int, stream, *args):
    """The C entry point `name` with the tensors' device current, on the given stream or that device's current one."""
    if index < 0:
        raise ValueError(f"the tensors lie on {like.device}, not on a GPU")
    if stream is not None and stream.device.index != index:
        raise ValueError(f"the stream belongs to {stream.device}, the tensors to {like.device}")
    fn = getattr(_lib or lib(), name)
    if index == torch.cuda.current_device():
        rc = fn(*args, _stream(stream))
    else:
        with torch.cuda.device(index):
            rc = fn(*args, _stream(stream))
    if rc:
        _check(name, rc)


def _ints(**sizes):
    """Refuses sizes that the C entry points' 32-bit integers would take the lower halves of."""
    for name, value in sizes.items():
        if not -2**31 <= value < 2**31:
            raise ValueError(f"{name} must be below 2^31, got {value}")


_I32, _F32 = torch.int32, torch.float32
_CODES = {torch.float32: F32, torch.bfloat16: BF16}


def embed_forward(tokens, table, out, scale: float = 1.0, stream=None):
    """out [..., d] = scale * table [n_classes, d] at tokens int32 [...]; zeros for tokens outside the table."""
    t, shape, whole, at = table.dtype, tokens.shape, table.shape, table.get_device()
    dtype = _CODES.get(t)
    if len(whole) != 2 or dtype is None:
        raise ValueError("table: [n_classes, d], float32 or bfloat16")
    V, d = whole
    if (V | d) >> 31:
        _ints(n_classes=V, d=d)
    _call_on("dsf_embed_forward", table, at, stream, _dense("tokens", tokens, shape, _I32, at),
             _dense("table", table, whole, t, at), dtype, tokens.numel(), V, d, scale,
             _dense("out", out, (*shape, d), t, at))


def embed_backward_workspace_size(n_tokens: int, d: int, n_classes: int) -> int:
    _ints(d=d, n_classes=n_classes)
    return lib().dsf_embed_backward_workspace_size(n_tokens, d, n_classes)


def embed_backward(tokens, dy, dtable, scale: float = 1.0, accumulate: bool = False, workspace=None, stream=None):
    """dtable [n_classes, d] (float32, or dy's dtype) = or += scale * the sums of dy [..., d] by token."""
    dtype, at = _dtype_code(dy), dy.get_device()
    if dtable.dim() != 2:
        raise ValueError("dtable: [n_classes, d]")
    V, d = dtable.shape
    if (V | d) >> 31:
        _ints(n_classes=V, d=d)
    n, shape = tokens.numel(), tokens.shape
    tp, yp = _dense("tokens", tokens, shape, _I32, at), _dense("dy", dy, (*shape, d), dy.dtype, at)
    gp = _dense("dtable", dtable, dtable.shape, dy.dtype, at, _F32)
    wp, wb, keep = _scratch(workspace, lambda: embed_backward_workspace_size(n, d, V), dy, stream)
    _call_on("dsf_embed_backward", dy, at, stream, tp, yp, dtype, n, V, d, scale, int(accumulate), gp,
             _dtype_code(dtable), wp, wb)


def norm_forward(x, w, out, b=None, eps: float = 1e-5, rms: bool = False, stream=None):
    """out = LayerNorm (rms: RMSNorm) of x [..., d] with gain w [d] and bias b [d] or None. out may be x."""
    t, at, shape = x.dtype, x.get_device(), x.shape
    dtype = _CODES.get(t)
    if dtype is None or not shape:
        raise ValueError("x: [..., d], float32 or bfloat16")
    d = shape[-1]
    if d >> 31:
        _ints(d=d)
    n = x.numel() // d if d else 0
    _call_on("dsf_norm_forward", x, at, stream, _dense("x", x, shape, t, at), _dense("w", w, (d,), t, at),
             _dense("b", b, (d,), t, at), dtype, n, d, eps, int(rms), _dense("out", out, shape, t, at))


def norm_backward_workspace_size(n_rows: int, d: int) -> int:
    _ints(d=d)
    return lib().dsf_norm_backward_workspace_size(n_rows, d)


def norm_backward(x, dy, w, dx, dw=None, db=None, add=None, eps: float = 1e-5, rms: bool = False, workspace=None,
                  stream=None):
    """dx [..., d] (or None) = add + the adjoint of norm_forward at dy; dw, db float32 [d] or None."""
    dtype, at, shape = _dtype_code(x), x.get_device(), x.shape
    d = shape[-1] if shape else 0
    if d >> 31:
        _ints(d=d)
    n = x.numel() // d if d else 0
    t = x.dtype
    ptrs = [_dense("x", x, shape, t, at), _dense("dy", dy, shape, t, at), _dense("w", w, (d,), t, at),
            _dense("add", add, shape, t, at)]
    outs = [_dense("dx", dx, shape, t, at), _dense("dw", dw, (d,), _F32, at), _dense("db", db, (d,), _F32, at)]
    wp, wb, keep = None, 0, None
    if workspace is not None or dw is not None or db is not None:
        wp, wb, keep = _scratch(workspace, lambda: norm_backward_workspace_size(n, d), x, stream)
    _call_on("dsf_norm_backward", x, at, stream, *ptrs, dtype, n, d, eps, int(rms), *outs, wp, wb)


def head_workspace_size(dtype: int, n_rows: int, d: int, n_classes: int, top: int = 0, gradients: bool = True) -> int:
    _ints(d=d, n_classes=n_classes, top=top)
    return lib().dsf_head_workspace_size(dtype, n_rows, d, n_classes, top, int(gradients))


def _head(name: str, h, w, lists, middle, top, row_weight, row_loss, total, dh, dw, grad_scale, mean, workspace, stream):
    dtype, at = _dtype_code(h), h.get_device()
    if h.dim() < 1 or w.dim() != 2:
        raise ValueError("h: [..., d], w: [n_classes, d]")
    V, d = w.shape
    if (V | d | top) >> 31:
        _ints(n_classes=V, d=d, top=top)
    rows = h.shape[:-1]
    n = h.numel() // d if d else 0
    t = h.dtype
    hp, wp = _dense("h", h, (*rows, d), t, at), _dense("w", w, w.shape, t, at)
    lp = [_dense(what, x, (*rows, *more), kind, at) for what, x, more, kind in lists]
    rw, rl = _dense("row_weight", row_weight, rows, _F32, at), _dense("row_loss", row_loss, rows, _F32, at)
    tp, dhp = _dense("total", total, (2,), _F32, at), _dense("dh", dh, h.shape, t, at)
    dwp = _dense("dw", dw, w.shape, t, at, _F32)
    grads = dh is not None or dw is not None
    sp, sb, keep = _scratch(workspace, lambda: head_workspace_size(dtype, n, d, V, top, grads), h, stream)
    _call_on(name, h, at, stream, hp, wp, dtype, n, d, V, *lp, *middle, rw, grad_scale, int(mean), rl, tp, dhp, dwp,
             _dtype_code(dw) if dw is not None else dtype, sp, sb)


def head_cross_entropy(h, w, targets, row_loss=None, total=None, dh=None, dw=None, row_weight=None,
                       grad_scale: float = 1.0, mean: bool = False, workspace=None, stream=None):
    """Cross entropy of the head w [n_classes, d] on rows h [..., d] with targets int32 [...] (others than classes: the
    row takes no part), and its gradients: row_loss, row_weight float32 [...], total float32 [2] (sum of weighted
    losses, sum of weights), dh as h, dw [n_classes, d] float32 or as w; None: not wanted (row_weight: ones)."""
    _head("dsf_head_cross_entropy", h, w, [("targets", targets, (), _I32)], (), 0, row_weight, row_loss, total, dh, dw,
          grad_scale, mean, workspace, stream)


def head_distill(h, w, top_classes, top_logits, temperature: float = 1.0, row_loss=None, total=None, dh=None, dw=None,
                 row_weight=None, grad_scale: float = 1.0, mean: bool = False, workspace=None, stream=None):
    """The head's loss against a teacher's top logits: top_classes int32, top_logits float32 [..., top]; entries of
    other numbers than classes are none. The rest as head_cross_entropy."""
    top = top_classes.shape[-1] if top_classes.dim() else 0
    _head("dsf_head_distill", h, w, [("top_classes", top_classes, (top,), _I32), ("top_logits", top_logits, (top,), _F32)],
          (top, temperature), top, row_weight, row_loss, total, dh, dw, grad_scale, mean, workspace, stream)


def timing_enable(max_records: int, kinds: Optional[Sequence[str]] = None):
    """Arm per-launch event timing for the named kernel classes (all if None)."""
    mask = (1 << len(KINDS)) - 1 if kinds is None else sum(1 << KINDS.index(k) for k in kinds)
    _check("dsf_timing_enable", lib().dsf_timing_enable(max_records, mask))


def timing_read(kind: str):
    n = ctypes.c_int(0)
    ms = ctypes.c_double(0.0)
    _check("dsf_timing_read", lib().dsf_timing_read(KINDS.index(kind), ctypes.addressof(n), ctypes.addressof(ms)))
    return n.value, ms.value


# ------------------------------------------------------ marshalling helpers

def make_desc(block: str, d_model: int, n_heads: int, n_kv_heads: int, head_dim: int, d_ff: int,
              rotary_dims: int, d_router: int, norm_eps: float, rope_theta: float) -> LayerDesc:
    code = {"neox_parallel": BLOCK_NEOX_PARALLEL, "qwen_seq": BLOCK_QWEN_SEQ}[block]
    return LayerDesc(code, d_model, n_heads, n_kv_heads, head_dim, d_ff, rotary_dims, d_router, norm_eps, 0.0,
                     rope_theta)


class DeviceLayer:
    """Keeps one layer's device tensors alive and exposes them as LayerWeights."""

    def __init__(self, tensors: dict, device):
        self.tensors = {}
        for name in _WEIGHT_FIELDS:
            if name in ("router_b2", "reserved"):
                continue
            t = tensors.get(name)
            self.tensors[name] = None if t is None else t.to(device).contiguous()
        self.router_b2 = float(tensors.get("router_b2", 0.0))
        kw = {n: _ptr(t) for n, t in self.tensors.items()}
        self.weights = LayerWeights(router_b2=self.router_b2, reserved=0.0, **kw)
