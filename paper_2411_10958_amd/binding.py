"""ctypes binding of libsageattn.so: argument marshalling only.

Every function here has the name and meaning of the C entry point it calls (see
include/sage_attn.h).  Tensors are torch tensors on the GPU; their device pointers are passed
through untouched.  There is no fallback: if the library cannot be loaded, every call raises.
"""
import ctypes
import os

import torch

SAGE_MODE_INT4_FP8, SAGE_MODE_INT8_FP8 = 0, 1
SAGE_DT_FP16, SAGE_DT_BF16 = 0, 1
SAGE_FLAG_SMOOTH_V = 1
SAGE_FLAG_NO_SMOOTH_K = 2
SAGE_FLAG_NO_SMOOTH_Q = 4
SAGE_FLAG_FP32_DELTA_S = 8
SAGE_FLAG_FP64_DELTA_S = 16
SAGE_FLAG_DIGIT_DELTA_S = 32
SAGE_GROUPS_LANE, SAGE_GROUPS_BLOCK, SAGE_GROUPS_FINE, SAGE_GROUPS_TOKEN, SAGE_GROUPS_TENSOR = 0, 1, 2, 3, 4
_GROUPS = {"lane": 0, "block": 1, "fine": 2, "token": 3, "tensor": 4, 0: 0, 1: 1, 2: 2, 3: 3, 4: 4}
_GROUP_SIZES = {0: (2, 16), 1: (2, 16), 2: (1, 4), 3: (1, 1), 4: (2, 16)}     # queries, keys per stored scale
SAGE_LAYOUT_HND, SAGE_LAYOUT_NHD = 0, 1
_LAYOUTS = {"HND": 0, "NHD": 1, 0: 0, 1: 1}
_MODES = {"int4_fp8": 0, "int8_fp8": 1, 0: 0, 1: 1}
SAGE_PV_E4M3, SAGE_PV_E5M2, SAGE_PV_INT8 = 0, 1, 2
_PV_FORMATS = {"e4m3": 0, "e5m2": 1, "int8": 2, 0: 0, 1: 1, 2: 2}

_PKG = os.path.dirname(os.path.abspath(__file__))
_LIB = None
# The current stream's handle without a Stream object (2.0 -> 0.1 us a call).  The name is private to torch: a build without it makes the object.
_current_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)


class SageError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        super().__init__(f"{where}: status {status} ({sage_status_string(status)})")


class sage_attn_args(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("out", ctypes.c_void_p),
                ("B", ctypes.c_int), ("H", ctypes.c_int), ("H_kv", ctypes.c_int),
                ("N", ctypes.c_int), ("d", ctypes.c_int),
                ("causal", ctypes.c_int), ("sm_scale", ctypes.c_float),
                ("mode", ctypes.c_int), ("dtype", ctypes.c_int), ("flags", ctypes.c_int), ("group_map", ctypes.c_int), ("N_kv", ctypes.c_int), ("layout", ctypes.c_int),
                ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t),
                ("stream", ctypes.c_void_p),
                ("cu_seqlens_q", ctypes.c_void_p), ("cu_seqlens_k", ctypes.c_void_p), ("lse", ctypes.c_void_p),
                ("pv_format", ctypes.c_int),
                ("k_mean_in", ctypes.c_void_p), ("v_scale_in", ctypes.c_void_p), ("kv_splits", ctypes.c_int)]


class sage_quant_out(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("q_codes", "k_codes", "v_codes", "q_scale", "k_scale",
                                              "v_scale", "k_mean", "q_mean", "delta_s", "v_mean")]


class sage_rope_args(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("q", "k", "q_out", "k_out")] + \
               [(n, ctypes.c_int) for n in ("B", "H", "H_kv", "N", "d", "rot_dim", "dtype", "layout", "interleaved", "inverse")] + \
               [("scale", ctypes.c_float), ("inv_freq", ctypes.c_void_p), ("positions", ctypes.c_void_p),
                ("positions_stride", ctypes.c_longlong), ("offset", ctypes.c_longlong)] + \
               [(n, ctypes.c_longlong * 3) for n in ("q_strides", "k_strides", "q_out_strides", "k_out_strides")] + [("stream", ctypes.c_void_p)]


class sage_attn_shared_prefix_args(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("q", "k_prefix", "v_prefix", "k", "v", "out", "kv_lens", "lse")] + \
               [(n, ctypes.c_int) for n in ("B", "H", "H_kv", "N", "N_prefix", "N_kv", "d", "causal")] + \
               [("sm_scale", ctypes.c_float), ("dtype", ctypes.c_int), ("layout", ctypes.c_int), ("workspace", ctypes.c_void_p),
                ("workspace_bytes", ctypes.c_size_t), ("stream", ctypes.c_void_p)]


class sage_attn_key_weights_args(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("q", "k", "lse", "weights_in", "weights", "kv_lens")] + \
               [(n, ctypes.c_int) for n in ("B", "H", "H_kv", "N", "N_kv", "d", "causal")] + \
               [("sm_scale", ctypes.c_float), ("dtype", ctypes.c_int), ("layout", ctypes.c_int), ("workspace", ctypes.c_void_p),
                ("workspace_bytes", ctypes.c_size_t), ("stream", ctypes.c_void_p)]


class sage_cache_evict_args(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("k", "v", "weights", "kv_lens", "k_out", "v_out", "weights_out", "kept", "lens_out")] + \
               [(n, ctypes.c_int) for n in ("B", "H_kv", "N_kv", "N_keep", "d", "sink", "recent", "dtype", "layout", "N_out")] + \
               [("stream", ctypes.c_void_p), ("clear", ctypes.c_int)]


class sage_qk_norm_rope_args(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("q", "k", "q_out", "k_out", "q_weight", "k_weight")] + \
               [(n, ctypes.c_int) for n in ("B", "H", "H_kv", "N", "d", "rot_dim", "dtype", "layout", "weight_type", "interleaved")] + \
               [("eps", ctypes.c_float), ("scale", ctypes.c_float), ("inv_freq", ctypes.c_void_p), ("positions", ctypes.c_void_p),
                ("positions_stride", ctypes.c_longlong), ("offset", ctypes.c_longlong)] + \
               [(n, ctypes.c_longlong * 3) for n in ("q_strides", "k_strides", "q_out_strides", "k_out_strides")] + [("stream", ctypes.c_void_p)]


class sage_qk_norm_rope_bwd_args(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("dq_out", "dk_out", "q", "k", "dq", "dk", "q_weight", "k_weight", "dq_weight", "dk_weight")] + \
               [(n, ctypes.c_int) for n in ("B", "H", "H_kv", "N", "d", "rot_dim", "dtype", "layout", "weight_type", "interleaved")] + \
               [("eps", ctypes.c_float), ("scale", ctypes.c_float), ("inv_freq", ctypes.c_void_p), ("positions", ctypes.c_void_p),
                ("positions_stride", ctypes.c_longlong), ("offset", ctypes.c_longlong)] + \
               [(n, ctypes.c_longlong * 3) for n in ("dq_out_strides", "dk_out_strides", "q_strides", "k_strides", "dq_strides", "dk_strides")] + \
               [("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t), ("stream", ctypes.c_void_p)]


class sage_cache_append_args(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("k", "v", "k_cache", "v_cache", "k_scale", "v_scale", "page_table", "kv_lens", "new_lens")] + \
               [(n, ctypes.c_int) for n in ("B", "H_kv", "N", "d", "n_pages", "page", "max_pages", "dtype", "layout")] + \
               [(n, ctypes.c_longlong * 3) for n in ("k_strides", "v_strides")] + [("stream", ctypes.c_void_p)]


class sage_attn_paged_args(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("q", "k_cache", "v_cache", "k_scale", "v_scale", "out", "page_table", "kv_lens", "q_lens", "lse")] + \
               [(n, ctypes.c_int) for n in ("B", "H", "H_kv", "N", "d", "n_pages", "page", "max_pages", "causal", "window", "sink")] + \
               [("sm_scale", ctypes.c_float), ("dtype", ctypes.c_int), ("layout", ctypes.c_int), ("clear", ctypes.c_int), ("workspace", ctypes.c_void_p),
                ("workspace_bytes", ctypes.c_size_t), ("stream", ctypes.c_void_p)]


def lib_path():
    """The in-tree library; SAGEATTN_LIB may name another build of the same sources."""
    return os.environ.get("SAGEATTN_LIB") or os.path.join(_PKG, "libsageattn.so")


def load_library():
    """Loads libsageattn.so from the package directory (built by paper_2411_10958_amd.build)."""
    global _LIB
    if _LIB is None:
        path = lib_path()
        if not os.path.exists(path):
            raise FileNotFoundError(f"{path} is missing: run `python -m paper_2411_10958_amd.build` "
                                    "(or __graft_entry__.build()) first")
        lib = ctypes.CDLL(path)
        P = ctypes.POINTER
        lib.sage_attn_workspace_bytes.restype = ctypes.c_size_t
        lib.sage_attn_workspace_bytes.argtypes = [P(sage_attn_args)]
        for name in ("sage_attn_fwd_ex", "sage_attn_prologue", "sage_attn_core", "sage_attn_fwd_static"):
            getattr(lib, name).restype = ctypes.c_int
            getattr(lib, name).argtypes = [P(sage_attn_args)]
        lib.sage_attn_fwd.restype = ctypes.c_int
        lib.sage_attn_fwd.argtypes = [ctypes.c_void_p] * 4 + [ctypes.c_int] * 5 + [ctypes.c_float, ctypes.c_int]
        lib.sage_attn_kv_splits.restype = ctypes.c_int
        lib.sage_attn_kv_splits.argtypes = [P(sage_attn_args)]
        lib.sage_attn_release.restype = None
        lib.sage_attn_kv_stats.restype = ctypes.c_int
        lib.sage_attn_kv_stats.argtypes = [P(sage_attn_args), ctypes.c_void_p, ctypes.c_void_p]
        lib.sage_attn_kv_stats_update.restype = ctypes.c_int
        lib.sage_attn_kv_stats_update.argtypes = [P(sage_attn_args), ctypes.c_void_p, ctypes.c_void_p, ctypes.c_longlong,
                                                  ctypes.c_void_p, ctypes.c_void_p]
        lib.sage_attn_quant.restype = ctypes.c_int
        lib.sage_attn_quant.argtypes = [P(sage_attn_args), P(sage_quant_out)]
        lib.sage_attn_debug_qk.restype = ctypes.c_int
        lib.sage_attn_debug_qk.argtypes = [P(sage_attn_args)] + [ctypes.c_int] * 4 + [ctypes.c_void_p]
        lib.sage_attn_debug_mfma_fp8.restype = ctypes.c_int
        lib.sage_attn_debug_mfma_fp8.argtypes = [ctypes.c_void_p] * 5
        for name in ("sage_rope", "sage_attn_shared_prefix", "sage_attn_key_weights", "sage_cache_evict", "sage_qk_norm_rope", "sage_qk_norm_rope_bwd",
                     "sage_cache_append", "sage_attn_paged"):
            getattr(lib, name).restype = ctypes.c_int
            getattr(lib, name).argtypes = [P(globals()[name + "_args"])]
        for name in ("sage_attn_shared_prefix", "sage_attn_key_weights", "sage_qk_norm_rope_bwd", "sage_attn_paged"):
            getattr(lib, name + "_workspace_bytes").restype = ctypes.c_size_t
            getattr(lib, name + "_workspace_bytes").argtypes = [P(globals()[name + "_args"])]
        lib.sage_rope_frequencies.restype = ctypes.c_int
        lib.sage_rope_frequencies.argtypes = [ctypes.c_int, ctypes.c_double, ctypes.c_int] + [ctypes.c_double] * 4 + [ctypes.c_void_p]
        lib.sage_status_string.restype = ctypes.c_char_p
        lib.sage_status_string.argtypes = [ctypes.c_int]
        _LIB = lib
    return _LIB


def sage_status_string(status):
    return load_library().sage_status_string(int(status)).decode()


def _check(status, where):
    if status != 0:
        raise SageError(status, where)


def _dtype_code(t):
    if t.dtype == torch.bfloat16:
        return SAGE_DT_BF16
    if t.dtype == torch.float16:
        return SAGE_DT_FP16
    raise TypeError(f"q, k, v must be float16 or bfloat16, got {t.dtype}")


def _ptr(t):
    return ctypes.c_void_p(t.data_ptr()) if t is not None else ctypes.c_void_p(0)


def make_args(q, k, v, out=None, causal=False, sm_scale=0.0, mode="int4_fp8", workspace=None, stream=None,
              smooth_v=False, group_map="lane", layout="HND", pv_format="e4m3", smooth_k=True, smooth_q=True,
              fp32_delta_s=False, kv_stats=None, kv_splits=0, delta_s=None):
    """delta_s: None (the library picks between the two exact forms of the Delta-S product), "digits", "fp64", or "fp32"
    (same as fp32_delta_s=True).
    Fills a sage_attn_args from torch tensors q [B,H,N,d], k/v [B,H_kv,N_kv,d] (layout "HND") or
    q [B,N,H,d], k/v [B,N_kv,H_kv,d] (layout "NHD"), contiguous, on the GPU.  `workspace` is a uint8 GPU tensor (or None); `stream` a torch.cuda.Stream (None = the
    current one)."""
    for t in (q, k, v):
        if not t.is_cuda or not t.is_contiguous() or t.dim() != 4:
            raise ValueError(f"{'qkv'[0 if t is q else 1 if t is k else 2]} must be a contiguous 4-D GPU tensor")
    dtype, qs, ks = q.dtype, q.shape, k.shape
    if ks != v.shape or k.dtype != dtype or v.dtype != dtype:
        raise ValueError("k and v must share shape; q, k, v must share dtype")
    nhd = _LAYOUTS[layout]
    if nhd:
        (B, N, H, d), (Bk, Nk, Hkv, dk) = qs, ks
    else:
        (B, H, N, d), (Bk, Hkv, Nk, dk) = qs, ks
    if Bk != B or dk != d:
        raise ValueError("k/v shape does not match q")
    if out is not None and (out.shape != qs or out.dtype != dtype or not out.is_contiguous()):
        raise ValueError("out must look like q")
    flags = SAGE_FLAG_SMOOTH_V if smooth_v else 0
    if not smooth_k:
        flags |= SAGE_FLAG_NO_SMOOTH_K
    if not smooth_q:
        flags |= SAGE_FLAG_NO_SMOOTH_Q
    if fp32_delta_s or delta_s is not None:
        flags |= ((SAGE_FLAG_FP32_DELTA_S if (fp32_delta_s or delta_s == "fp32") else 0) |
                  (SAGE_FLAG_FP64_DELTA_S if delta_s == "fp64" else 0) | (SAGE_FLAG_DIGIT_DELTA_S if delta_s == "digits" else 0))
    km_ptr = vs_ptr = None
    if kv_stats is not None:       # (k_mean, v_scale) float32 GPU tensors [B, H_kv, d], e.g. from sage_attn_kv_stats
        km, vs = kv_stats
        for name, t in (("k_mean", km), ("v_scale", vs)):
            # (the first extent is the batch size, or the number of sequences of a packed batch)
            if not t.is_cuda or t.dtype != torch.float32 or not t.is_contiguous() or t.dim() != 3 or \
                    tuple(t.shape[1:]) != (Hkv, d):
                raise ValueError(f"kv_stats: {name} must be a contiguous float32 GPU tensor of shape [B, H_kv, d]")
        km_ptr, vs_ptr = km.data_ptr(), vs.data_ptr()
    if stream is not None:
        raw_stream = stream.cuda_stream
    else:
        raw_stream = _current_raw_stream(q.get_device())
    # the fields in their order: one call instead of an attribute at a time (the whole of this function 5.2 -> 2.0 us)
    return sage_attn_args(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr() if out is not None else 0,
                          B, H, Hkv, N, d, int(bool(causal)), float(sm_scale), _MODES[mode], _dtype_code(q), flags,
                          _GROUPS[group_map], Nk, nhd,
                          workspace.data_ptr() if workspace is not None else 0,
                          workspace.numel() * workspace.element_size() if workspace is not None else 0,
                          raw_stream, 0, 0, 0, _PV_FORMATS[pv_format], km_ptr, vs_ptr, int(kv_splits))


def sage_attn_workspace_bytes(args):
    return int(load_library().sage_attn_workspace_bytes(ctypes.byref(args)))


def sage_attn_kv_splits(args):
    """Key chunks per query tile the attention kernel will use for these arguments (in their workspace, where they have one)."""
    return int(load_library().sage_attn_kv_splits(ctypes.byref(args)))


def _alloc_workspace(args, device):
    need = sage_attn_workspace_bytes(args)
    if need == 0:
        raise SageError(load_library().sage_attn_prologue(ctypes.byref(args)) or -1, "sage_attn_workspace_bytes")
    ws = torch.empty(need, dtype=torch.uint8, device=device)
    args.workspace, args.workspace_bytes = ws.data_ptr(), need
    return ws


def sage_attn_fwd_ex(q, k, v, out=None, causal=False, sm_scale=0.0, mode="int4_fp8", workspace=None, stream=None,
                     smooth_v=False, group_map="lane", layout="HND", cu_seqlens_q=None, cu_seqlens_k=None,
                     max_seqlen_q=None, max_seqlen_k=None, return_lse=False, pv_format="e4m3", smooth_k=True,
                     smooth_q=True, fp32_delta_s=False, kv_stats=None, kv_splits=0, delta_s=None):
    """Whole forward pass.  Returns `out` (allocated if not given).  With cu_seqlens_q the batch is a packed
    variable-length one (see make_varlen_args) and `layout` is ignored.  With return_lse the result is
    (out, lse): lse float32 [B, H, N], or [H, total_q] for a variable-length batch."""
    if out is None:
        out = torch.empty_like(q)
    if cu_seqlens_q is not None:
        a = make_varlen_args(q, k, v, out, cu_seqlens_q, cu_seqlens_k, max_seqlen_q, max_seqlen_k, causal=causal,
                             sm_scale=sm_scale, mode=mode, workspace=workspace, stream=stream, smooth_v=smooth_v,
                             group_map=group_map, pv_format=pv_format, smooth_k=smooth_k, smooth_q=smooth_q,
                             fp32_delta_s=fp32_delta_s, kv_stats=kv_stats, kv_splits=kv_splits, delta_s=delta_s)
    else:
        a = make_args(q, k, v, out, causal, sm_scale, mode, workspace, stream, smooth_v, group_map, layout, pv_format,
                      smooth_k, smooth_q, fp32_delta_s, kv_stats, kv_splits, delta_s)
    lse = None
    if return_lse:
        shape = (a.H, q.shape[0]) if cu_seqlens_q is not None else (a.B, a.H, a.N)
        lse = torch.empty(shape, dtype=torch.float32, device=q.device)
        a.lse = lse.data_ptr()
    keep = _alloc_workspace(a, q.device) if workspace is None else workspace
    if workspace is None and stream is not None:
        keep.record_stream(stream)   # allocated on the current stream, used on another one
    _check(load_library().sage_attn_fwd_ex(ctypes.byref(a)), "sage_attn_fwd_ex")
    del keep  # torch's caching allocator keeps the block alive for work already queued on its streams
    return (out, lse) if return_lse else out


def sage_attn_fwd_static(q, k, v, out, causal=False, sm_scale=0.0, mode="int4_fp8", stream=None, **kw):
    """The forward pass on the library's built-in workspace (no allocation anywhere: `out` is the caller's).
    **kw as make_args."""
    a = make_args(q, k, v, out, causal, sm_scale, mode, None, stream, **kw)
    _check(load_library().sage_attn_fwd_static(ctypes.byref(a)), "sage_attn_fwd_static")
    return out


def make_varlen_args(q, k, v, out, cu_seqlens_q, cu_seqlens_k=None, max_seqlen_q=None, max_seqlen_k=None, **kw):
    """sage_attn_args of a packed variable-length batch: q / out [total_q, H, d], k / v [total_k, H_kv, d],
    cu_seqlens_* int32 GPU tensors [B + 1] (cu_seqlens_k None = the query one), max_seqlen_* the longest
    sequence (taken from the prefix sums, with a device-to-host copy, when not given).  **kw as make_args."""
    for name, t in (("q", q), ("k", k), ("v", v)):
        if not t.is_cuda or not t.is_contiguous() or t.dim() != 3:
            raise ValueError(f"{name} must be a contiguous 3-D GPU tensor")
    for name, t in (("cu_seqlens_q", cu_seqlens_q), ("cu_seqlens_k", cu_seqlens_k)):
        if t is not None and (not t.is_cuda or t.dtype != torch.int32 or t.dim() != 1 or not t.is_contiguous()):
            raise ValueError(f"{name} must be a contiguous 1-D int32 GPU tensor")
    if cu_seqlens_k is not None and cu_seqlens_k.numel() != cu_seqlens_q.numel():
        raise ValueError("cu_seqlens_q and cu_seqlens_k must have the same length")
    B = cu_seqlens_q.numel() - 1
    if B < 1:
        raise ValueError("cu_seqlens_q must hold at least two entries")
    if max_seqlen_q is None:
        max_seqlen_q = int((cu_seqlens_q[1:] - cu_seqlens_q[:-1]).max().item())
    if max_seqlen_k is None:
        ck = cu_seqlens_k if cu_seqlens_k is not None else cu_seqlens_q
        max_seqlen_k = int((ck[1:] - ck[:-1]).max().item())
    # the struct is filled through [1, tokens, heads, d] views; B, N, N_kv are then set for the packed batch
    a = make_args(q.unsqueeze(0), k.unsqueeze(0), v.unsqueeze(0), None if out is None else out.unsqueeze(0),
                  layout="NHD", **kw)
    a.B, a.N, a.N_kv = B, max(int(max_seqlen_q), 1), max(int(max_seqlen_k), 1)
    a.cu_seqlens_q = cu_seqlens_q.data_ptr()
    a.cu_seqlens_k = cu_seqlens_k.data_ptr() if cu_seqlens_k is not None else 0
    return a


def sage_attn_prologue(args):
    _check(load_library().sage_attn_prologue(ctypes.byref(args)), "sage_attn_prologue")


def sage_attn_core(args):
    _check(load_library().sage_attn_core(ctypes.byref(args)), "sage_attn_core")


def sage_attn_fwd(q, k, v, out, causal=False, sm_scale=0.0, mode="int4_fp8"):
    """The plain C signature: bf16, H_kv == H, default stream, library-owned workspace."""
    B, H, N, d = q.shape
    _check(load_library().sage_attn_fwd(_ptr(q), _ptr(k), _ptr(v), _ptr(out), B, H, N, d, int(bool(causal)),
                                         float(sm_scale), _MODES[mode]), "sage_attn_fwd")
    return out


def sage_attn_kv_stats(k, v, layout="HND", pv_format="e4m3", cu_seqlens_k=None, max_seqlen_k=None, workspace=None,
                       stream=None):
    """mean(K) and delta_V alone (the statistics pass of the preprocessing): returns (k_mean, v_scale), float32
    [B, H_kv, d] each, in the form the `kv_stats` argument of the other calls takes.  With cu_seqlens_k, k and v are
    packed [total_k, H_kv, d] tensors and B is the number of sequences."""
    if cu_seqlens_k is not None:
        a = make_varlen_args(k, k, v, None, cu_seqlens_k, cu_seqlens_k, max_seqlen_k, max_seqlen_k, workspace=workspace,
                             stream=stream, pv_format=pv_format)
    else:
        a = make_args(k, k, v, None, workspace=workspace, stream=stream, layout=layout, pv_format=pv_format)
    keep = _alloc_workspace(a, k.device) if workspace is None else workspace
    km = torch.empty((a.B, a.H_kv, a.d), dtype=torch.float32, device=k.device)
    vs = torch.empty_like(km)
    st = load_library().sage_attn_kv_stats(ctypes.byref(a), ctypes.c_void_p(km.data_ptr()), ctypes.c_void_p(vs.data_ptr()))
    if st != 0:
        raise SageError(st, "sage_attn_kv_stats")
    del keep
    return km, vs


def sage_attn_kv_stats_update(k_new, v_new, state, layout="HND", pv_format="e4m3", workspace=None, stream=None):
    """Running statistics of a growing K / V.  k_new, v_new: the new tokens [B, H_kv, n_new, d]; state: None for the
    first chunk, else what the previous call returned.  Returns (k_mean, v_scale, state): the statistics of everything
    accumulated so far (as `kv_stats` takes them) and the updated state (k_sum float64, v_absmax float32, token count)."""
    a = make_args(k_new, k_new, v_new, None, workspace=workspace, stream=stream, layout=layout, pv_format=pv_format)
    keep = _alloc_workspace(a, k_new.device) if workspace is None else workspace
    shape = (a.B, a.H_kv, a.d)
    if state is None:
        ks = torch.empty(shape, dtype=torch.float64, device=k_new.device)
        vm = torch.empty(shape, dtype=torch.float32, device=k_new.device)
        n_before = 0
    else:
        ks, vm, n_before = state
    km = torch.empty(shape, dtype=torch.float32, device=k_new.device)
    vs = torch.empty_like(km)
    st = load_library().sage_attn_kv_stats_update(ctypes.byref(a), ctypes.c_void_p(ks.data_ptr()), ctypes.c_void_p(vm.data_ptr()),
                                                  ctypes.c_longlong(n_before), ctypes.c_void_p(km.data_ptr()),
                                                  ctypes.c_void_p(vs.data_ptr()))
    if st != 0:
        raise SageError(st, "sage_attn_kv_stats_update")
    del keep
    return km, vs, (ks, vm, n_before + a.N_kv)


def sage_attn_release():
    load_library().sage_attn_release()


def sage_attn_quant(q, k, v, causal=False, sm_scale=0.0, mode="int4_fp8", workspace=None, want=None,
                    smooth_v=False, group_map="lane", pv_format="e4m3", smooth_k=True, smooth_q=True,
                    fp32_delta_s=False, kv_stats=None, delta_s=None):
    """Preprocessing only; returns (dict of torch tensors in plain layouts, args, workspace)."""
    a = make_args(q, k, v, None, causal, sm_scale, mode, workspace, smooth_v=smooth_v, group_map=group_map,
                  pv_format=pv_format, smooth_k=smooth_k, smooth_q=smooth_q, fp32_delta_s=fp32_delta_s,
                  kv_stats=kv_stats, delta_s=delta_s)
    ws = _alloc_workspace(a, q.device) if workspace is None else workspace
    B, H, N, d = q.shape
    Hkv, Nk = k.shape[1], k.shape[2]
    dev = q.device
    int4 = _MODES[mode] == 0
    nqb = (N + 127) // 128
    qg, kg = _GROUP_SIZES[_GROUPS[group_map]]
    bufs = dict(
        q_codes=torch.empty((B, H, N, d), dtype=torch.int8, device=dev),
        k_codes=torch.empty((B, Hkv, Nk, d), dtype=torch.int8, device=dev),
        v_codes=torch.empty((B, Hkv, Nk, d), dtype=torch.uint8, device=dev),
        q_scale=torch.empty((B, H, (N + qg - 1) // qg), dtype=torch.float32, device=dev),
        k_scale=torch.empty((B, Hkv, (Nk + kg - 1) // kg), dtype=torch.float32, device=dev),
        v_scale=torch.empty((B, Hkv, d), dtype=torch.float32, device=dev),
        k_mean=torch.empty((B, Hkv, d), dtype=torch.float32, device=dev),
    )
    if int4:
        bufs["q_mean"] = torch.empty((B, H, nqb, d), dtype=torch.float32, device=dev)
        bufs["delta_s"] = torch.empty((B, H, nqb, Nk), dtype=torch.float32, device=dev)
    if smooth_v:
        bufs["v_mean"] = torch.empty((B, Hkv, d), dtype=torch.float32, device=dev)
    if want is not None:
        bufs = {n: t for n, t in bufs.items() if n in want}
    o = sage_quant_out()
    for n, _ in sage_quant_out._fields_:
        setattr(o, n, bufs[n].data_ptr() if n in bufs else 0)
    _check(load_library().sage_attn_quant(ctypes.byref(a), ctypes.byref(o)), "sage_attn_quant")
    return bufs, a, ws


def sage_attn_debug_qk(args, b, h, q_tile, kv_block, device="cuda"):
    out = torch.empty((128, 64), dtype=torch.int32, device=device)
    _check(load_library().sage_attn_debug_qk(ctypes.byref(args), b, h, q_tile, kv_block, _ptr(out)), "sage_attn_debug_qk")
    return out


def sage_attn_debug_mfma_fp8(a_codes, b_codes, c_in):
    """One v_mfma_f32_32x32x64_f8f6f4: a_codes, b_codes uint8 [64, 32] (E4M3), c_in float32 [64, 16]."""
    d = torch.empty_like(c_in)
    s = torch.cuda.current_stream(c_in.device).cuda_stream
    _check(load_library().sage_attn_debug_mfma_fp8(_ptr(a_codes), _ptr(b_codes), _ptr(c_in), _ptr(d), s),
           "sage_attn_debug_mfma_fp8")
    return d


# ---- operators around the attention calls: rotary positions, a shared prefix, key weights, eviction ----

SAGE_ROPE_PLAIN, SAGE_ROPE_LINEAR, SAGE_ROPE_BASE, SAGE_ROPE_PARTS = 0, 1, 2, 3
SAGE_WEIGHT_FP32, SAGE_WEIGHT_SAME = 0, 1
SAGE_CLEAR_OUT, SAGE_CLEAR_LSE = 1, 2
_ROPE_SCALINGS = {"plain": 0, "linear": 1, "base": 2, "parts": 3, 0: 0, 1: 1, 2: 2, 3: 3}


def _gpu_of(name, t):
    """The index of the GPU that t is on."""
    index = t.get_device()
    if index < 0:
        raise ValueError(f"{name} must be a GPU tensor")
    return index


def _need(name, t, index, dtype, shape=None):
    """Raises unless t is a contiguous tensor of that type (and shape) on GPU `index`."""
    if t.get_device() != index or t.dtype != dtype or (shape is not None and t.shape != shape) or not t.is_contiguous():
        _refuse(name, t, index, dtype, shape)


def _refuse(name, t, index, dtype, shape):
    if t.get_device() != index:
        raise ValueError(f"{name} must be on GPU {index} like the other tensors, is on {t.device}")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    raise ValueError(f"{name} must be contiguous")


def _new(shape, dtype, index, stream, make=torch.empty):
    """An output or a workspace from torch's allocator.  For another stream it is allocated (and filled) there: the block may have been
    another tensor's, and what is still queued for that one is ordered with the stream that it came from."""
    if stream is None:
        return make(shape, dtype=dtype, device=index)
    with torch.cuda.stream(stream):
        t = make(shape, dtype=dtype, device=index)
    t.record_stream(torch.cuda.current_stream(index))        # the caller goes on with it here
    return t


def _stream_on(index, stream):
    """The raw stream of a call on GPU `index`.  A kernel started on another GPU's stream would run there, on these addresses."""
    if stream is None:
        return _current_raw_stream(index)
    if stream.device_index != index:
        raise ValueError(f"stream must be one of GPU {index} like the tensors, is of GPU {stream.device_index}")
    return stream.cuda_stream


def _whole(x, bits):
    """A whole number for a C field of so many bits: one that does not fit becomes the field's end, which the call refuses, instead of another number."""
    x = int(x)
    return max(-(1 << bits - 1), min(x, (1 << bits - 1) - 1))


def _address(t):
    return 0 if t is None else t.data_ptr()


def _call(name, args, index):
    """One entry point with its argument structure, on the device of its tensors."""
    f = getattr(load_library(), name)
    if torch.cuda.current_device() == index:
        status = f(ctypes.byref(args))
    else:
        with torch.cuda.device(index):
            status = f(ctypes.byref(args))
    if status != 0:
        raise SageError(status, name)


def _own_workspace(name, args, index, workspace, stream):
    """Points args at `workspace`, or at a new one.  The result has to live until the call is enqueued."""
    if workspace is None:
        need = getattr(load_library(), name + "_workspace_bytes")(ctypes.byref(args))
        if need == 0:
            return None
        workspace = _new(need, torch.uint8, index, stream)
        args.workspace, args.workspace_bytes = workspace.data_ptr(), need
        return workspace
    if workspace.get_device() != index or not workspace.is_contiguous():
        raise ValueError(f"workspace must be a contiguous tensor on GPU {index}")
    args.workspace, args.workspace_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    return workspace


def _sizes(name, x, nhd):
    """B, heads, tokens, d of a 4-D tensor."""
    if x.dim() != 4:
        raise ValueError(f"{name} must have 4 dimensions, got {x.dim()}")
    B, m, n, d = x.shape
    return (B, n, m, d) if nhd else (B, m, n, d)


def sage_rope_frequencies(rot_dim, base=10000.0, scaling="plain", factor=1.0, original_length=0.0, low=1.0, high=32.0, device=None):
    """The rot_dim / 2 frequencies, in radians per position, for sage_rope: a float64 tensor on `device` (None: the current GPU).
    scaling: "plain"; for contexts `factor` times longer than trained for, "linear" (all divided by it), "base" (the base raised so that
    the slowest is divided by it) or "parts" (those that turn `high` times or more in original_length tokens kept, `low` times or fewer
    divided, linear between)."""
    out = (ctypes.c_double * max(int(rot_dim) // 2, 1))()
    _check(load_library().sage_rope_frequencies(int(rot_dim), float(base), _ROPE_SCALINGS[scaling], float(factor), float(original_length),
                                                float(low), float(high), ctypes.cast(out, ctypes.c_void_p)), "sage_rope_frequencies")
    return torch.tensor(list(out), dtype=torch.float64, device="cuda" if device is None else device)


def sage_rope(q, k=None, inv_freq=None, positions=None, offset=0, interleaved=False, inverse=False, scale=1.0, layout="HND", q_out=None,
              k_out=None, stream=None):
    """Rotary positions of q and k in one launch: the first 2 * len(inv_freq) channels of every row are turned, the others copied.
    q [B, H, N, d], k [B, H_kv, N, d] or None (layout "HND"; tokens outside heads with "NHD"), or packed [tokens, heads, d] with positions
    [tokens].  Any strides will do while the channels are contiguous.  positions: int32 [N] or [B, N] (None: 0 .. N - 1), `offset` is
    added.  inverse turns back; with the same scale (0 stands for 1) that is the gradient.  q_out, k_out may be q and k.  Returns
    q_out, or (q_out, k_out)."""
    if inv_freq is None:
        raise ValueError("inv_freq is needed (see sage_rope_frequencies)")
    dtype, index = _dtype_code(q), _gpu_of("q", q)
    raw_stream = _stream_on(index, stream)
    packed = q.dim() == 3
    if not packed and q.dim() != 4:
        raise ValueError(f"q must have 4 dimensions, or 3 if packed, got {q.dim()}")
    nhd = 1 if packed else _LAYOUTS[layout]
    B, H, N, d = (1, q.shape[1], q.shape[0], q.shape[2]) if packed else _sizes("q", q, nhd)
    Hkv = 0
    if k is not None:
        if k.get_device() != index or k.dtype != q.dtype or k.dim() != q.dim():
            raise ValueError("k must have the type, device and number of dimensions of q")
        Bk, Hkv, Nk, dk = (1, k.shape[1], k.shape[0], k.shape[2]) if packed else _sizes("k", k, nhd)
        if (Bk, Nk, dk) != (B, N, d):
            raise ValueError("k shape does not match q")
    elif k_out is not None:
        raise ValueError("k_out without k")
    if q.numel() == 0 or (k is not None and Hkv == 0):
        raise ValueError("q or k is empty")
    _need("inv_freq", inv_freq, index, torch.float64)
    if inv_freq.dim() != 1:
        raise ValueError("inv_freq must have one dimension")
    if positions is not None:
        _need("positions", positions, index, torch.int32)
        if positions.shape != (N,) and positions.shape != (B, N):
            raise ValueError(f"positions must have shape ({N},) or ({B}, {N}), got {tuple(positions.shape)}")
    elif packed:
        raise ValueError("a packed batch needs positions")
    outs = []
    for name, x, y in (("q_out", q, q_out), ("k_out", k, k_out)):
        if x is None:
            y = None
        elif y is None:
            y = _new(x.shape, x.dtype, index, stream)
        elif y.get_device() != index or y.dtype != q.dtype or y.shape != x.shape:
            raise ValueError(f"{name} must have the type, shape and device of its input")
        outs.append(y)
    a = sage_rope_args(q.data_ptr(), _address(k), outs[0].data_ptr(), _address(outs[1]), B, H, Hkv, N, d, 2 * inv_freq.numel(), dtype, nhd,
                       int(bool(interleaved)), int(bool(inverse)), float(scale), inv_freq.data_ptr(), _address(positions),
                       N if positions is not None and positions.dim() == 2 else 0, _whole(offset, 64))
    a.stream = raw_stream
    for t, st in ((q, a.q_strides), (k, a.k_strides), (outs[0], a.q_out_strides), (outs[1], a.k_out_strides)):
        if t is None or t.is_contiguous():
            continue                            # (all zero: contiguous)
        s = t.stride()
        if s[-1] != 1:
            raise ValueError("the channels of a row must be contiguous")
        if packed:
            s = (0,) + s[:-1]
        st[0], st[1], st[2] = (s[0], s[2], s[1]) if nhd else s[:3]
        if not any(st):
            raise ValueError("one row expanded over all others is not supported (strides of zero stand for a contiguous tensor)")
    _call("sage_rope", a, index)
    return outs[0] if k is None else tuple(outs)


def _shared_prefix_args(q, k_prefix, v_prefix, k, v, kv_lens, out, causal, sm_scale, layout, stream):
    dtype, dt, index, nhd = _dtype_code(q), q.dtype, _gpu_of("q", q), _LAYOUTS[layout]
    raw_stream = _stream_on(index, stream)
    B, H, N, d = _sizes("q", q, nhd)
    _need("q", q, index, dt)
    if (k_prefix is None) != (v_prefix is None) or (k is None) != (v is None) or (k is None and k_prefix is None):
        raise ValueError("a prefix, own keys and values, or both are needed, each with its values")
    P = Nk = 0
    Hkv = None
    if k_prefix is not None:
        if k_prefix.dim() != 3:
            raise ValueError(f"k_prefix must have 3 dimensions, got {k_prefix.dim()}")
        P, Hkv, dp = k_prefix.shape if nhd else (k_prefix.shape[1], k_prefix.shape[0], k_prefix.shape[2])
        _need("k_prefix", k_prefix, index, dt)
        _need("v_prefix", v_prefix, index, dt, k_prefix.shape)
        if dp != d:
            raise ValueError("the prefix does not match q")
    if k is not None:
        Bk, Hk, Nk, dk = _sizes("k", k, nhd)
        _need("k", k, index, dt)
        _need("v", v, index, dt, k.shape)
        if Bk != B or dk != d or (Hkv is not None and Hk != Hkv):
            raise ValueError("k does not match q or the prefix")
        Hkv = Hk
    if kv_lens is not None:
        _need("kv_lens", kv_lens, index, torch.int32, (B,))
    if out is not None:
        _need("out", out, index, dt, q.shape)
    return sage_attn_shared_prefix_args(q.data_ptr(), _address(k_prefix), _address(v_prefix), _address(k), _address(v), _address(out), _address(kv_lens), 0,
                                        B, H, Hkv, N, P, Nk, d, int(bool(causal)), float(sm_scale), dtype, nhd, 0, 0,
                                        raw_stream)


def sage_attn_shared_prefix_workspace_bytes(args):
    """The size of the workspace to hand to sage_attn_shared_prefix, 0 if it needs none.  args: a sage_attn_shared_prefix_args, of which the sizes, dtype
    (SAGE_DT_*), layout (0 HND, 1 NHD) and causal are looked at."""
    return int(load_library().sage_attn_shared_prefix_workspace_bytes(ctypes.byref(args)))


def sage_attn_shared_prefix(q, k_prefix, v_prefix, k=None, v=None, kv_lens=None, out=None, causal=True, sm_scale=0.0, layout="HND",
                            return_lse=False, workspace=None, stream=None):
    """16-bit attention of q [B, H, N, d] over a prefix [H_kv, P, d] that all sequences share (None: none), then over each
    sequence's own k, v [B, H_kv, N_kv, d] (None: none), of which the first kv_lens (int32 [B]; None: all) are in use.  Layout "NHD":
    tokens outside heads in all of them.  causal masks the own keys, aligned to the last query and key in use.  Returns out, or
    (out, lse) with lse float32 [B, H, N]."""
    a = _shared_prefix_args(q, k_prefix, v_prefix, k, v, kv_lens, out, causal, sm_scale, layout, stream)
    index, lse = q.get_device(), None
    if out is None:
        out = _new(q.shape, q.dtype, index, stream)
        a.out = out.data_ptr()
    if return_lse:
        lse = _new((a.B, a.H, a.N), torch.float32, index, stream)
        a.lse = lse.data_ptr()
    keep = _own_workspace("sage_attn_shared_prefix", a, index, workspace, stream)
    _call("sage_attn_shared_prefix", a, index)
    del keep
    return (out, lse) if return_lse else out


def sage_attn_key_weights_workspace_bytes(args):
    """The size of the workspace to hand to sage_attn_key_weights, 0 if it needs none.  args: a sage_attn_key_weights_args, of which the sizes, dtype
    (SAGE_DT_*), layout (0 HND, 1 NHD) and causal are looked at."""
    return int(load_library().sage_attn_key_weights_workspace_bytes(ctypes.byref(args)))


def sage_attn_key_weights(q, k, lse, weights_in=None, weights=None, kv_lens=None, causal=True, sm_scale=0.0, layout="HND", workspace=None,
                          stream=None):
    """What each key of k [B, H_kv, N_kv, d] has received of the attention of q [B, H, N, d] with log-sum-exp lse (float32 [B, H, N], as the
    attention calls return it), summed over the queries of its KV head and added to weights_in.  Returns weights, float32
    [B, H_kv, N_kv]; may be weights_in.  Entries behind kv_lens keep what they hold (zeros if the result is allocated here)."""
    dtype, index, nhd = _dtype_code(q), _gpu_of("q", q), _LAYOUTS[layout]
    raw_stream = _stream_on(index, stream)
    B, H, N, d = _sizes("q", q, nhd)
    Bk, Hkv, Nk, dk = _sizes("k", k, nhd)
    _need("q", q, index, q.dtype)
    _need("k", k, index, q.dtype)
    if Bk != B or dk != d:
        raise ValueError("k does not match q")
    _need("lse", lse, index, torch.float32, (B, H, N))
    shape = (B, Hkv, Nk)
    if weights_in is not None:
        _need("weights_in", weights_in, index, torch.float32, shape)
    if kv_lens is not None:
        _need("kv_lens", kv_lens, index, torch.int32, (B,))
    if weights is None:
        weights = _new(shape, torch.float32, index, stream, torch.empty if kv_lens is None else torch.zeros)
    else:
        _need("weights", weights, index, torch.float32, shape)
    a = sage_attn_key_weights_args(q.data_ptr(), k.data_ptr(), lse.data_ptr(), _address(weights_in), weights.data_ptr(), _address(kv_lens),
                                   B, H, Hkv, N, Nk, d, int(bool(causal)), float(sm_scale), dtype, nhd, 0, 0,
                                   raw_stream)
    keep = _own_workspace("sage_attn_key_weights", a, index, workspace, stream)
    _call("sage_attn_key_weights", a, index)
    del keep
    return weights


def sage_cache_evict(k, v, weights, n_keep, sink=0, recent=0, kv_lens=None, layout="HND", k_out=None, v_out=None, weights_out=None, kept=None,
                     lens_out=None, stream=None, room=None):
    """Cuts a cache k, v [B, H_kv, N_kv, d] to n_keep tokens per KV head: the first `sink` and the last `recent` of those in use
    (kv_lens, int32 [B]; None: all) and the ones of largest weight (float32 [B, H_kv, N_kv]) between.  Returns (k_out, v_out,
    weights_out, kept, lens_out): the rows kept, in their order, their weights, which they were (int32 [B, H_kv, n_keep]) and how many
    (int32 [B]); what stands behind them keeps what it held (zeros where the output is allocated here).  k_out, v_out and weights_out
    have room for `room` tokens (None: n_keep), so that the cache can go on growing there."""
    dtype, dt, index, nhd = _dtype_code(k), k.dtype, _gpu_of("k", k), _LAYOUTS[layout]
    raw_stream = _stream_on(index, stream)
    B, Hkv, Nk, d = _sizes("k", k, nhd)
    _need("k", k, index, dt)
    _need("v", v, index, dt, k.shape)
    n_keep = int(n_keep)
    if n_keep < 1:
        raise ValueError("n_keep must be at least 1")
    room = n_keep if room is None else int(room)
    if room < n_keep:
        raise ValueError(f"room must be n_keep, {n_keep}, or more, got {room}")
    _need("weights", weights, index, torch.float32, (B, Hkv, Nk))
    if kv_lens is not None:
        _need("kv_lens", kv_lens, index, torch.int32, (B,))
    # Places behind what is kept: where all outputs are made here, the call itself writes zeros there, and nothing is filled before
    behind = kv_lens is not None or room > Nk or room > n_keep
    clear = behind and k_out is None and v_out is None and weights_out is None and kept is None
    make = torch.zeros if behind and not clear else torch.empty
    rows = (B, room, Hkv, d) if nhd else (B, Hkv, room, d)
    outs = []
    for name, t, shape, want in (("k_out", k_out, rows, dt), ("v_out", v_out, rows, dt), ("weights_out", weights_out, (B, Hkv, room), torch.float32),
                                 ("kept", kept, (B, Hkv, n_keep), torch.int32), ("lens_out", lens_out, (B,), torch.int32)):
        if t is None:
            t = _new(shape, want, index, stream, make if name != "lens_out" else torch.empty)
        else:
            _need(name, t, index, want, shape)
        outs.append(t)
    a = sage_cache_evict_args(k.data_ptr(), v.data_ptr(), weights.data_ptr(), _address(kv_lens), *[t.data_ptr() for t in outs],
                              B, Hkv, Nk, n_keep, d, _whole(sink, 32), _whole(recent, 32), dtype, nhd, room,
                              raw_stream, int(clear))
    _call("sage_cache_evict", a, index)
    return tuple(outs)


def _set_strides(field, t, packed, nhd):
    """Batch, head and token strides of t into a field of an argument structure; left at zeros for a contiguous tensor."""
    s = t.stride()
    if s[-1] != 1 and t.shape[-1] != 1:
        raise ValueError("the channels of a row must be contiguous")
    if packed:
        s = (0,) + s[:-1]
    field[0], field[1], field[2] = (s[0], s[2], s[1]) if nhd else s[:3]
    if not any(field):
        raise ValueError("one row expanded over all others is not supported (strides of zero stand for a contiguous tensor)")


def _check_norm_rope(q, k, inv_freq, q_weight, k_weight, positions, index, packed, nhd, sizes):
    """Raises for what a call of sage_qk_norm_rope or its gradient got that does not go together."""
    B, H, N, d = sizes
    if not packed and q.dim() != 4:
        raise ValueError(f"q must have 4 dimensions, or 3 if packed, got {q.dim()}")
    if k is not None:
        if k.get_device() != index or k.dtype != q.dtype or k.dim() != q.dim():
            raise ValueError("k must have the type, device and number of dimensions of q")
        Bk, Hkv, Nk, dk = (1, k.shape[1], k.shape[0], k.shape[2]) if packed else _sizes("k", k, nhd)
        if (Bk, Nk, dk) != (B, N, d):
            raise ValueError("k shape does not match q")
    elif k_weight is not None:
        raise ValueError("k_weight without k")
    if q.numel() == 0 or (k is not None and k.numel() == 0):
        raise ValueError("q or k is empty")
    if inv_freq is not None:
        _need("inv_freq", inv_freq, index, torch.float64)
        if inv_freq.dim() != 1 or inv_freq.numel() == 0:
            raise ValueError("inv_freq must have one dimension and a frequency at least")
    if positions is not None:
        _need("positions", positions, index, torch.int32)
        if positions.shape != (N,) and positions.shape != (B, N):
            raise ValueError(f"positions must have shape ({N},) or ({B}, {N}), got {tuple(positions.shape)}")
    elif packed and inv_freq is not None:
        raise ValueError("a packed batch needs positions")
    if q_weight is not None:
        _need("q_weight", q_weight, index, q_weight.dtype, (d,))
    if k_weight is not None:
        _need("k_weight", k_weight, index, k_weight.dtype if q_weight is None else q_weight.dtype, (d,))
    weight = q_weight if q_weight is not None else k_weight
    if weight is not None and weight.dtype != torch.float32 and weight.dtype != q.dtype:
        raise TypeError(f"the weights must both be float32 or both {q.dtype}, got {weight.dtype}")


def _norm_rope_sizes(q, layout):
    """packed, token-major, (B, H, N, d)."""
    shape = q.shape
    if len(shape) == 3:
        return True, 1, (1, shape[1], shape[0], shape[2])
    nhd = _LAYOUTS[layout]
    if len(shape) != 4:
        raise ValueError(f"q must have 4 dimensions, or 3 if packed, got {len(shape)}")
    return False, nhd, (shape[0], shape[2], shape[1], shape[3]) if nhd else tuple(shape)


def _output_like(name, x, y, index, stream):
    if x is None:
        return None
    if y is None:
        return _new(x.shape, x.dtype, index, stream)
    if y.get_device() != index or y.dtype != x.dtype or y.shape != x.shape:
        raise ValueError(f"{name} must have the type, shape and device of its input")
    return y


def _grad_of(name, x, g, index):
    """Raises unless g, the gradient of an output, goes with the input x."""
    if g.get_device() != index or g.dtype != x.dtype or g.shape != x.shape:
        raise ValueError(f"{name} must have the type, shape and device of its input")


def _weight_grad(name, w, g, shape, index, stream):
    """Room for a weight's gradient, as given or new; None for a weight that is not there."""
    if w is None:
        if g is not None:
            raise ValueError(f"{name} without its weight")
        return None
    if g is None:
        return _new(shape, torch.float32, index, stream)
    _need(name, g, index, torch.float32, shape)
    return g


def _norm_rope_common(q, k, inv_freq, q_weight, k_weight, eps, positions, offset, interleaved, scale, packed, sizes, nhd, dtype):
    """The fields from B on that the two argument structures share."""
    weight = q_weight if q_weight is not None else k_weight
    return (*sizes[:2], 0 if k is None else k.shape[1] if packed or not nhd else k.shape[2], *sizes[2:], 0 if inv_freq is None else 2 * inv_freq.numel(), dtype, nhd,
            0 if weight is None or weight.dtype == torch.float32 else 1, 1 if interleaved else 0, eps, scale, _address(inv_freq), _address(positions),
            sizes[2] if positions is not None and positions.dim() == 2 else 0, _whole(offset, 64))


def sage_qk_norm_rope(q, k=None, inv_freq=None, q_weight=None, k_weight=None, eps=1e-6, positions=None, offset=0, interleaved=False, scale=1.0, layout="HND",
                      q_out=None, k_out=None, stream=None):
    """Every row of q and k divided by the root of its mean square (plus eps), times the weight of its channels (float32 or the tensors' type, [d]; None:
    ones), and its first 2 * len(inv_freq) channels turned as sage_rope does (inv_freq None: none), in one pass.  q [B, H, N, d], k [B, H_kv, N, d] or None
    (layout "HND"; tokens outside heads with "NHD"), or packed [tokens, heads, d]; any strides will do while the channels are contiguous.  q_out, k_out may be q and
    k.  Returns q_out, or (q_out, k_out)."""
    dtype, index = _dtype_code(q), _gpu_of("q", q)
    packed, nhd, sizes = _norm_rope_sizes(q, layout)
    raw_stream = _stream_on(index, stream)
    _check_norm_rope(q, k, inv_freq, q_weight, k_weight, positions, index, packed, nhd, sizes)
    if k is None and k_out is not None:
        raise ValueError("k_out without k")
    q_out, k_out = _output_like("q_out", q, q_out, index, stream), _output_like("k_out", k, k_out, index, stream)
    a = sage_qk_norm_rope_args(q.data_ptr(), _address(k), q_out.data_ptr(), _address(k_out), _address(q_weight), _address(k_weight),
                               *_norm_rope_common(q, k, inv_freq, q_weight, k_weight, eps, positions, offset, interleaved, scale, packed, sizes, nhd, dtype))
    a.stream = raw_stream
    if not q.is_contiguous():
        _set_strides(a.q_strides, q, packed, nhd)
    if not q_out.is_contiguous():
        _set_strides(a.q_out_strides, q_out, packed, nhd)
    if k is not None:
        if not k.is_contiguous():
            _set_strides(a.k_strides, k, packed, nhd)
        if not k_out.is_contiguous():
            _set_strides(a.k_out_strides, k_out, packed, nhd)
    _call("sage_qk_norm_rope", a, index)
    return q_out if k is None else (q_out, k_out)


def sage_qk_norm_rope_bwd_workspace_bytes(args):
    """The size of the workspace to hand to sage_qk_norm_rope_bwd, 0 if it needs none.  args: a sage_qk_norm_rope_bwd_args, of which the sizes, dtype, layout, k and
    whether the weights' gradients are wanted are looked at."""
    return int(load_library().sage_qk_norm_rope_bwd_workspace_bytes(ctypes.byref(args)))


def sage_qk_norm_rope_bwd(dq_out, q, dk_out=None, k=None, inv_freq=None, q_weight=None, k_weight=None, eps=1e-6, positions=None, offset=0, interleaved=False,
                          scale=1.0, layout="HND", dq=None, dk=None, dq_weight=None, dk_weight=None, workspace=None, stream=None):
    """The gradient of sage_qk_norm_rope: from that of its outputs, dq_out and dk_out, and its inputs, (dq, dk, dq_weight, dk_weight); dk is None
    without k.  The weights' are float32 [d], and None for a weight that is None.  dq may be dq_out, and dk dk_out."""
    dtype, index = _dtype_code(q), _gpu_of("q", q)
    packed, nhd, sizes = _norm_rope_sizes(q, layout)
    raw_stream = _stream_on(index, stream)
    _check_norm_rope(q, k, inv_freq, q_weight, k_weight, positions, index, packed, nhd, sizes)
    if (k is None) != (dk_out is None) or (k is None and dk is not None):
        raise ValueError("k, its gradient and that of its output go together")
    _grad_of("dq_out", q, dq_out, index)
    if k is not None:
        _grad_of("dk_out", k, dk_out, index)
    dq, dk = _output_like("dq", q, dq, index, stream), _output_like("dk", k, dk, index, stream)
    dq_weight = _weight_grad("dq_weight", q_weight, dq_weight, sizes[3:], index, stream)
    dk_weight = _weight_grad("dk_weight", k_weight, dk_weight, sizes[3:], index, stream)
    a = sage_qk_norm_rope_bwd_args(dq_out.data_ptr(), _address(dk_out), q.data_ptr(), _address(k), dq.data_ptr(), _address(dk), _address(q_weight), _address(k_weight),
                                   _address(dq_weight), _address(dk_weight),
                                   *_norm_rope_common(q, k, inv_freq, q_weight, k_weight, eps, positions, offset, interleaved, scale, packed, sizes, nhd, dtype))
    a.stream = raw_stream
    if not dq_out.is_contiguous():
        _set_strides(a.dq_out_strides, dq_out, packed, nhd)
    if not q.is_contiguous():
        _set_strides(a.q_strides, q, packed, nhd)
    if not dq.is_contiguous():
        _set_strides(a.dq_strides, dq, packed, nhd)
    if k is not None:
        if not dk_out.is_contiguous():
            _set_strides(a.dk_out_strides, dk_out, packed, nhd)
        if not k.is_contiguous():
            _set_strides(a.k_strides, k, packed, nhd)
        if not dk.is_contiguous():
            _set_strides(a.dk_strides, dk, packed, nhd)
    keep = _own_workspace("sage_qk_norm_rope_bwd", a, index, workspace, stream)
    _call("sage_qk_norm_rope_bwd", a, index)
    del keep
    return dq, dk, dq_weight, dk_weight


_E4M3, _E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu


def _paged_cache(k_cache, v_cache, k_scale, v_scale, page_table, index, B, Hkv, d):
    """The arrays of a cache in pages, checked: (pages, tokens of a page, pages of a sequence)."""
    if k_cache.dim() != 4 or page_table.dim() != 2:
        raise ValueError("k_cache must have 4 dimensions and page_table 2")
    shape = k_cache.shape
    pages, heads, page, dc = shape
    if heads != Hkv or dc != d:
        raise ValueError(f"k_cache must have shape [pages, {Hkv}, page, {d}], got {tuple(shape)}")
    if page % 32 != 0 or page == 0:
        raise ValueError(f"a page must hold a multiple of 32 tokens, got {page}")
    blocks = (pages, heads, page // 32)
    _need("k_cache", k_cache, index, _E4M3)
    _need("v_cache", v_cache, index, _E4M3, shape)
    _need("k_scale", k_scale, index, _E8M0, blocks)
    _need("v_scale", v_scale, index, _E8M0, blocks)
    of_one = page_table.shape[1]
    _need("page_table", page_table, index, torch.int32, (B, of_one))
    return pages, page, of_one


def sage_cache_append(k, v, k_cache, v_cache, k_scale, v_scale, page_table, kv_lens=None, new_lens=None, layout="HND", stream=None):
    """Writes new tokens k, v [B, H_kv, N, d] (layout "NHD": tokens outside heads; any strides will do while the channels are contiguous) into a cache in 8
    bits and pages: k_cache, v_cache float8_e4m3fn [pages, H_kv, page, d], k_scale, v_scale float8_e8m0fnu [pages, H_kv, page / 32], one power of two for
    each block of 32 tokens; page_table int32 [B, pages of a sequence], a number that is no page stands for none.  kv_lens (int32 [B]; None: the
    table's capacity): tokens of each sequence with the new ones, of which the first new_lens (int32 [B]; None: N) rows are the last."""
    dtype, index, nhd = _dtype_code(k), _gpu_of("k", k), _LAYOUTS[layout]
    raw_stream = _stream_on(index, stream)
    B, Hkv, N, d = _sizes("k", k, nhd)
    if v.get_device() != index or v.dtype != k.dtype or v.shape != k.shape:
        raise ValueError("v must have the type, shape and device of k")
    pages, page, max_pages = _paged_cache(k_cache, v_cache, k_scale, v_scale, page_table, index, B, Hkv, d)
    if kv_lens is not None:
        _need("kv_lens", kv_lens, index, torch.int32, (B,))
    if new_lens is not None:
        _need("new_lens", new_lens, index, torch.int32, (B,))
    a = sage_cache_append_args(k.data_ptr(), v.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), page_table.data_ptr(),
                               _address(kv_lens), _address(new_lens), B, Hkv, N, d, pages, page, max_pages, dtype, nhd)
    a.stream = raw_stream
    if not k.is_contiguous():
        _set_strides(a.k_strides, k, False, nhd)
    if not v.is_contiguous():
        _set_strides(a.v_strides, v, False, nhd)
    _call("sage_cache_append", a, index)


def sage_attn_paged_workspace_bytes(args):
    """The size of the workspace to hand to sage_attn_paged, 0 if it needs none.  args: a sage_attn_paged_args, of which the sizes, dtype, layout, causal, window and
    sink are looked at."""
    return int(load_library().sage_attn_paged_workspace_bytes(ctypes.byref(args)))


def sage_attn_paged(q, k_cache, v_cache, k_scale, v_scale, page_table, kv_lens=None, q_lens=None, out=None, causal=True, window=0, sink=0, sm_scale=0.0,
                    layout="HND", return_lse=False, workspace=None, stream=None):
    """Attention of q [B, H, N, d] over a cache in 8 bits and pages (see sage_cache_append), of which the first kv_lens tokens (int32 [B]; None: the table's
    capacity) of each sequence are in use.  The first q_lens queries (int32 [B]; None: N) of a sequence are there, the last of them aligned with its last
    token if causal; the others' rows keep what they held (zeros where the output is allocated here).  window > 0: a query sees the last `window` tokens up
    to its own and the first `sink`.  Returns out, or (out, lse) with lse float32 [B, H, N]."""
    dtype, index, nhd = _dtype_code(q), _gpu_of("q", q), _LAYOUTS[layout]
    raw_stream = _stream_on(index, stream)
    B, H, N, d = _sizes("q", q, nhd)
    _need("q", q, index, q.dtype)
    Hkv = k_cache.shape[1] if k_cache.dim() == 4 else 0
    pages, page, max_pages = _paged_cache(k_cache, v_cache, k_scale, v_scale, page_table, index, B, Hkv, d)
    clear = 0                                   # rows behind q_lens: what is made here the call fills with zeros there
    if kv_lens is not None:
        _need("kv_lens", kv_lens, index, torch.int32, (B,))
    if q_lens is not None:
        _need("q_lens", q_lens, index, torch.int32, (B,))
        clear = (SAGE_CLEAR_OUT if out is None else 0) | SAGE_CLEAR_LSE
    if out is None:
        out = _new(q.shape, q.dtype, index, stream)
    else:
        _need("out", out, index, q.dtype, q.shape)
    lse = _new((B, H, N), torch.float32, index, stream) if return_lse else None
    a = sage_attn_paged_args(q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), out.data_ptr(), page_table.data_ptr(),
                             _address(kv_lens), _address(q_lens), _address(lse), B, H, Hkv, N, d, pages, page, max_pages, 1 if causal else 0,
                             _whole(window, 32), _whole(sink, 32), sm_scale, dtype, nhd, clear, 0, 0, raw_stream)
    keep = _own_workspace("sage_attn_paged", a, index, workspace, stream)
    _call("sage_attn_paged", a, index)
    del keep
    return (out, lse) if return_lse else out
