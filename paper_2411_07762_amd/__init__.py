"""Python binding of libaser.so: the MI355X implementation of ASER's per-layer calibration path.

Argument marshalling only.  Every function has the name and the meaning of the C entry point
declared in include/aser.h; tensors are torch tensors on the GPU (torch provides device memory
and the stream, nothing else) or raw integer device addresses.  There is no CPU fallback: if
the HIP library has not been built, importing the entry points raises.
"""
from __future__ import annotations

import ctypes
import functools
import os
from typing import Optional

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libaser.so")

ASER_OK = 0
ASER_ERR_INVALID_ARG = 1
ASER_ERR_SHAPE = 2
ASER_ERR_DTYPE = 3
ASER_ERR_NOT_SPD = 4
ASER_ERR_NO_CONVERGE = 5
ASER_ERR_WORKSPACE = 6
ASER_ERR_HIP = 7

ASER_DTYPE_BF16 = 0
ASER_DTYPE_F32 = 1
ASER_PRECISION_AUTO = 0
ASER_PRECISION_FAST = 1
ASER_PRECISION_EXACT = 2
ASER_CODES_INT8 = 0
ASER_CODES_INT4_PACKED = 1
ASER_KV_BF16 = 0
ASER_KV_INT8 = 1

EXPORTS = (
    "aser_status_string", "aser_create", "aser_destroy", "aser_last_error", "aser_set_workspace", "aser_set_precision",
    "aser_workspace_bytes", "aser_gram_accumulate", "aser_smooth_outliers", "aser_smooth_outliers_noalloc",
    "aser_quantize_rtn",
    "aser_whiten", "aser_error_reconstruct", "aser_svd_plan", "aser_quantize_act_rtn",
    "aser_spectrum_workspace_bytes", "aser_singular_values", "aser_select_rank", "aser_effective_rank",
    "aser_output_error_workspace_bytes", "aser_layer_output_error",
    "aser_forward_workspace_bytes", "aser_compensated_forward", "aser_mfma_rate_probe",
    "aser_error_reconstruct_enqueue", "aser_finish", "aser_calibrate_layers", "aser_pick_concurrent_streams",
    "aser_layer_workspace_bytes", "aser_smoothed_weight", "aser_quant_target",
    "aser_kv_append", "aser_paged_attention", "aser_paged_attention_workspace_bytes",
    "aser_adapter_forward", "aser_adapter_workspace_bytes",
    "aser_mx4_quantize", "aser_mx4_forward", "aser_mx4_forward_workspace_bytes",
    "aser_route_experts", "aser_route_workspace_bytes", "aser_expert_forward", "aser_expert_forward_workspace_bytes", "aser_expert_combine",
)


class aser_svd_opts(ctypes.Structure):
    _fields_ = [("block", ctypes.c_int32), ("max_iter", ctypes.c_int32), ("seed", ctypes.c_uint32)]


class aser_layer_desc(ctypes.Structure):
    """Mirror of the C struct of the same name (one layer of aser_calibrate_layers)."""
    _vp, _i64, _i32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32
    _fields_ = [("X", _vp), ("x_dtype", _i32), ("clear_stats", _i32), ("rows", _i64), ("ldx", _i64),
                ("G", _vp), ("ldg", _i64), ("abs_sum", _vp), ("count", _vp),
                ("W", _vp), ("m", _i64), ("n", _i64), ("ldw", _i64), ("f", _i32), ("bits", _i32),
                ("idx", _vp), ("mdiag", _vp),
                ("layout", _i32), ("r", _i32), ("codes", _vp), ("scales", _vp), ("T", _vp), ("ldt", _i64),
                ("damp", ctypes.c_float), ("stats_from", _i32), ("S", _vp), ("lds", _i64),
                ("opts", ctypes.POINTER(aser_svd_opts)), ("L_A", _vp), ("L_B", _vp), ("sigma", _vp),
                ("err", ctypes.c_double), ("n_iter", _i32), ("status", _i32)]


class aser_kv_cache(ctypes.Structure):
    """Mirror of the C struct of the same name; KvCache fills one from tensors."""
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
                ("n_pages", ctypes.c_int64), ("page_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64),
                ("slot_stride", ctypes.c_int64), ("dtype", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("n_kv", ctypes.c_int32), ("head_dim", ctypes.c_int32)]


class aser_kv_batch(ctypes.Structure):
    """Mirror of the C struct of the same name; KvBatch fills one from tensors."""
    _fields_ = [("start", ctypes.c_void_p), ("kv_len", ctypes.c_void_p), ("pages", ctypes.c_void_p), ("ld_pages", ctypes.c_int64),
                ("tokens", ctypes.c_int64), ("n_seq", ctypes.c_int32), ("max_new", ctypes.c_int32), ("max_kv", ctypes.c_int32)]


class aser_qk_opts(ctypes.Structure):
    _fields_ = [("rope_cos", ctypes.c_void_p), ("rope_sin", ctypes.c_void_p), ("q_norm", ctypes.c_void_p), ("k_norm", ctypes.c_void_p),
                ("n_pos", ctypes.c_int64), ("rot_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("eps", ctypes.c_float)]


class aser_mx4(ctypes.Structure):
    """Mirror of the C struct of the same name; Mx4 fills one from tensors."""
    _fields_ = [("codes", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("rows", ctypes.c_int64), ("n", ctypes.c_int64), ("count", ctypes.c_int32)]


class aser_expert_plan(ctypes.Structure):
    """Mirror of the C struct of the same name; ExpertPlan fills one from tensors."""
    _fields_ = [("ids", ctypes.c_void_p), ("weights", ctypes.c_void_p), ("offsets", ctypes.c_void_p), ("order", ctypes.c_void_p),
                ("place", ctypes.c_void_p), ("rows", ctypes.c_int64), ("top_k", ctypes.c_int32), ("n_experts", ctypes.c_int32)]


class aser_route_opts(ctypes.Structure):
    _fields_ = [("sigmoid", ctypes.c_int32), ("n_groups", ctypes.c_int32), ("top_groups", ctypes.c_int32), ("group_top", ctypes.c_int32),
                ("renormalize", ctypes.c_int32), ("scale", ctypes.c_float)]


class AserError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__("aser status %d (%s): %s" % (status, status_string(status), message))
        self.status = status


_lib = None


def load_library() -> ctypes.CDLL:
    """Loads libaser.so built in-tree by paper_2411_07762_amd.build; raises if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError("libaser.so is not built: run `python -m paper_2411_07762_amd.build` "
                           "(there is no CPU fallback for the HIP path)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i64, i32, f32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_float
    lib.aser_status_string.restype = ctypes.c_char_p
    lib.aser_status_string.argtypes = [ctypes.c_int]
    lib.aser_create.restype = ctypes.c_int
    lib.aser_create.argtypes = [ctypes.POINTER(vp), ctypes.c_int, vp]
    lib.aser_destroy.restype = ctypes.c_int
    lib.aser_destroy.argtypes = [vp]
    lib.aser_last_error.restype = ctypes.c_char_p
    lib.aser_last_error.argtypes = [vp]
    lib.aser_set_workspace.restype = ctypes.c_int
    lib.aser_set_workspace.argtypes = [vp, vp, ctypes.c_size_t]
    lib.aser_set_precision.restype = ctypes.c_int
    lib.aser_set_precision.argtypes = [vp, ctypes.c_int]
    lib.aser_workspace_bytes.restype = ctypes.c_size_t
    lib.aser_workspace_bytes.argtypes = [i64, i64, i32, ctypes.POINTER(aser_svd_opts)]
    lib.aser_gram_accumulate.restype = ctypes.c_int
    lib.aser_gram_accumulate.argtypes = [vp, vp, ctypes.c_int, i64, i64, i64, vp, i64, vp, vp]
    lib.aser_smooth_outliers.restype = ctypes.c_int
    lib.aser_smooth_outliers.argtypes = [vp, vp, i64, i64, i64, vp, vp, i32, vp, vp, vp, vp]
    lib.aser_smooth_outliers_noalloc.restype = ctypes.c_int
    lib.aser_smooth_outliers_noalloc.argtypes = lib.aser_smooth_outliers.argtypes
    lib.aser_quantize_rtn.restype = ctypes.c_int
    lib.aser_quantize_rtn.argtypes = [vp, vp, i64, i64, i64, vp, vp, i32, i32, i32, vp, vp, vp, i64]
    lib.aser_smoothed_weight.restype = ctypes.c_int
    lib.aser_smoothed_weight.argtypes = [vp, vp, i64, i64, i64, vp, i32, vp, i64]
    lib.aser_quant_target.restype = ctypes.c_int
    lib.aser_quant_target.argtypes = [vp, vp, i64, i64, i64, vp, vp, i64, vp, i64]
    lib.aser_whiten.restype = ctypes.c_int
    lib.aser_whiten.argtypes = [vp, vp, i64, i64, vp, f32, vp, i64, ctypes.POINTER(ctypes.c_int32)]
    lib.aser_error_reconstruct.restype = ctypes.c_int
    lib.aser_error_reconstruct.argtypes = [vp, vp, i64, i64, i64, vp, i64, i32, vp, i32, ctypes.POINTER(aser_svd_opts),
                                           vp, vp, vp, ctypes.POINTER(ctypes.c_double),
                                           ctypes.POINTER(ctypes.c_int32)]
    lib.aser_error_reconstruct_enqueue.restype = ctypes.c_int
    lib.aser_error_reconstruct_enqueue.argtypes = lib.aser_error_reconstruct.argtypes[:-2]
    lib.aser_finish.restype = ctypes.c_int
    lib.aser_finish.argtypes = [vp, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int32)]
    lib.aser_calibrate_layers.restype = ctypes.c_int
    lib.aser_calibrate_layers.argtypes = [ctypes.POINTER(vp), i32, ctypes.POINTER(aser_layer_desc), i32]
    lib.aser_layer_workspace_bytes.restype = ctypes.c_size_t
    lib.aser_layer_workspace_bytes.argtypes = [ctypes.POINTER(aser_layer_desc)]
    lib.aser_pick_concurrent_streams.restype = ctypes.c_int
    lib.aser_pick_concurrent_streams.argtypes = [i32, ctypes.POINTER(vp), i32, i32, ctypes.POINTER(i32), ctypes.POINTER(i32)]
    lib.aser_svd_plan.restype = ctypes.c_int
    lib.aser_svd_plan.argtypes = [i64, i64, i32, ctypes.POINTER(aser_svd_opts), ctypes.POINTER(ctypes.c_int32),
                                  ctypes.POINTER(ctypes.c_int32)]
    lib.aser_spectrum_workspace_bytes.restype = ctypes.c_size_t
    lib.aser_spectrum_workspace_bytes.argtypes = [i64, i64, i32]
    lib.aser_singular_values.restype = ctypes.c_int
    lib.aser_singular_values.argtypes = [vp, vp, i64, i64, i64, vp, i64, vp]
    lib.aser_select_rank.restype = ctypes.c_int
    lib.aser_select_rank.argtypes = [vp, vp, i64, ctypes.c_double, ctypes.POINTER(ctypes.c_int32),
                                     ctypes.POINTER(ctypes.c_double)]
    lib.aser_effective_rank.restype = ctypes.c_int
    lib.aser_effective_rank.argtypes = [vp, vp, i64, ctypes.c_double, ctypes.POINTER(ctypes.c_double)]
    lib.aser_output_error_workspace_bytes.restype = ctypes.c_size_t
    lib.aser_output_error_workspace_bytes.argtypes = [i64, i64, i64, i32]
    lib.aser_layer_output_error.restype = ctypes.c_int
    lib.aser_layer_output_error.argtypes = [vp, vp, i64, i64, i64, vp, ctypes.c_int, i64, i64, vp, vp, i32, vp, vp, vp, i32,
                                            i32, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_double)]
    lib.aser_forward_workspace_bytes.restype = ctypes.c_size_t
    lib.aser_forward_workspace_bytes.argtypes = [i64, i64, i64, i32]
    lib.aser_compensated_forward.restype = ctypes.c_int
    lib.aser_compensated_forward.argtypes = [vp, vp, vp, i64, i64, vp, i32, vp, i64, vp, vp, i32, i32, vp, i64]
    lib.aser_quantize_act_rtn.restype = ctypes.c_int
    lib.aser_quantize_act_rtn.argtypes = [vp, vp, ctypes.c_int, i64, i64, i64, vp, i32, vp, vp]
    cache, batch = ctypes.POINTER(aser_kv_cache), ctypes.POINTER(aser_kv_batch)
    lib.aser_kv_append.restype = ctypes.c_int
    lib.aser_kv_append.argtypes = [vp, vp, i64, i32, vp, i64, vp, i64, i32, ctypes.POINTER(aser_qk_opts), cache, batch, vp, i64]
    lib.aser_paged_attention_workspace_bytes.restype = ctypes.c_size_t
    lib.aser_paged_attention_workspace_bytes.argtypes = [cache, batch, i32]
    lib.aser_paged_attention.restype = ctypes.c_int
    lib.aser_paged_attention.argtypes = [vp, vp, i64, i32, cache, batch, f32, i32, i32, vp, i64]
    lib.aser_adapter_workspace_bytes.restype = ctypes.c_size_t
    lib.aser_adapter_workspace_bytes.argtypes = [i64, i64, i64, i32]
    lib.aser_adapter_forward.restype = ctypes.c_int
    lib.aser_adapter_forward.argtypes = [vp, vp, ctypes.c_int, i64, i64, i64, vp, vp, vp, vp, i32, i32, i64, vp, i64, vp, i64]
    mx, plan = ctypes.POINTER(aser_mx4), ctypes.POINTER(aser_expert_plan)
    lib.aser_mx4_quantize.restype = ctypes.c_int
    lib.aser_mx4_quantize.argtypes = [vp, vp, ctypes.c_int, i64, vp, mx, vp, i64]
    lib.aser_mx4_forward_workspace_bytes.restype = ctypes.c_size_t
    lib.aser_mx4_forward_workspace_bytes.argtypes = [i64, i64, i64, i32]
    lib.aser_mx4_forward.restype = ctypes.c_int
    lib.aser_mx4_forward.argtypes = [vp, mx, mx, vp, vp, i32, i32, vp, i32, i64]
    lib.aser_route_workspace_bytes.restype = ctypes.c_size_t
    lib.aser_route_workspace_bytes.argtypes = [i64, i32, i32]
    lib.aser_route_experts.restype = ctypes.c_int
    lib.aser_route_experts.argtypes = [vp, vp, i32, i64, vp, ctypes.POINTER(aser_route_opts), plan]
    lib.aser_expert_forward_workspace_bytes.restype = ctypes.c_size_t
    lib.aser_expert_forward_workspace_bytes.argtypes = [i64, i64, i64, i32, i32]
    lib.aser_expert_forward.restype = ctypes.c_int
    lib.aser_expert_forward.argtypes = [vp, mx, mx, plan, i32, vp, vp, i32, i32, vp, i32, i64]
    lib.aser_expert_combine.restype = ctypes.c_int
    lib.aser_expert_combine.argtypes = [vp, vp, i32, i64, i64, plan, vp, i64, vp, i32, i64]
    lib.aser_mfma_rate_probe.restype = ctypes.c_int
    lib.aser_mfma_rate_probe.argtypes = [vp, i32, i32, i32, ctypes.POINTER(ctypes.c_double)]
    _lib = lib
    return lib


def status_string(status: int) -> str:
    return load_library().aser_status_string(int(status)).decode()


# ----------------------------------------------------------------------------------- marshalling
def _ptr(t) -> Optional[int]:
    """Device address of a tensor (or a raw int address, or None)."""
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _ld(t, cols: int) -> int:
    if isinstance(t, int) or t is None:
        return cols
    if t.dim() == 1:
        return cols
    if t.stride(-1) != 1:
        raise ValueError("matrices must be row-major with unit column stride")
    return t.stride(0)


_DTYPE_CODES = {}


def _dtype_code(t) -> int:
    if not _DTYPE_CODES:
        import torch
        _DTYPE_CODES.update({torch.bfloat16: ASER_DTYPE_BF16, torch.float32: ASER_DTYPE_F32})
    code = _DTYPE_CODES.get(t.dtype)
    if code is None:
        raise TypeError("activations must be bfloat16 or float32")
    return code


_TYPES = None


def _types():
    """torch's bfloat16, float32 and int32, kept in _TYPES (importing this package does not import torch)."""
    global _TYPES
    import torch
    _TYPES = torch.bfloat16, torch.float32, torch.int32
    return _TYPES


class Context:
    """Owns an aser_ctx bound to a device and a HIP stream (torch's current stream by default)."""

    def __init__(self, device: int = 0, stream: Optional[int] = None):
        self._lib = load_library()
        if stream is None:
            import torch
            stream = torch.cuda.current_stream(device).cuda_stream
        h = ctypes.c_void_p()
        st = self._lib.aser_create(ctypes.byref(h), int(device), ctypes.c_void_p(stream))
        if st != ASER_OK:
            raise AserError(st, "aser_create failed")
        self.handle = h
        self.device = device
        self._ws = None
        self._ws_bytes = 0

    def close(self):
        if self.handle:
            self._lib.aser_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def set_precision(self, mode: int):
        self.check(self._lib.aser_set_precision(self.handle, int(mode)))

    def last_error(self) -> str:
        return self._lib.aser_last_error(self.handle).decode()

    def check(self, status: int):
        if status != ASER_OK:
            raise AserError(status, self.last_error())

    def ensure_workspace(self, nbytes: int):
        """Allocates (with torch) and binds a workspace of at least nbytes."""
        import torch
        nbytes = (int(nbytes) + 255) // 256 * 256
        if self._ws is None or self._ws_bytes < nbytes:
            new = torch.empty(nbytes + 256, dtype=torch.uint8, device="cuda:%d" % self.device)
            base = new.data_ptr()
            off = (-base) % 256
            # the old tensor stays alive until the library has read what it left pending in it
            st = self._lib.aser_set_workspace(self.handle, ctypes.c_void_p(base + off), nbytes)
            self._ws, self._ws_bytes = new, nbytes
            self.check(st)


def aser_workspace_bytes(m: int, n: int, r: int, opts: Optional[aser_svd_opts] = None) -> int:
    return int(load_library().aser_workspace_bytes(m, n, r, ctypes.byref(opts) if opts is not None else None))


def aser_set_workspace(ctx: Context, dev_ptr, nbytes: int) -> int:
    return ctx._lib.aser_set_workspace(ctx.handle, ctypes.c_void_p(_ptr(dev_ptr)), int(nbytes))


def aser_gram_accumulate(ctx: Context, X, G, abs_sum=None, count=None, *, rows=None, n=None, ldx=None, ldg=None,
                         x_dtype=None) -> int:
    rows = X.shape[0] if rows is None else rows
    n = X.shape[1] if n is None else n
    return ctx._lib.aser_gram_accumulate(
        ctx.handle, _ptr(X), _dtype_code(X) if x_dtype is None else x_dtype, rows, n,
        _ld(X, n) if ldx is None else ldx, _ptr(G), _ld(G, n) if ldg is None else ldg, _ptr(abs_sum), _ptr(count))


def aser_smooth_outliers(ctx: Context, W, abs_sum, count, f: int, idx, mdiag, W_o=None, score=None, *, m=None, n=None,
                         ldw=None) -> int:
    m = W.shape[0] if m is None else m
    n = W.shape[1] if n is None else n
    return ctx._lib.aser_smooth_outliers(ctx.handle, _ptr(W), m, n, _ld(W, n) if ldw is None else ldw, _ptr(abs_sum),
                                         _ptr(count), f, _ptr(idx), _ptr(mdiag), _ptr(W_o), _ptr(score))


def aser_smooth_outliers_noalloc(ctx: Context, W, abs_sum, count, f: int, idx, mdiag, W_o=None, score=None, *, m=None,
                                 n=None, ldw=None) -> int:
    m = W.shape[0] if m is None else m
    n = W.shape[1] if n is None else n
    return ctx._lib.aser_smooth_outliers_noalloc(ctx.handle, _ptr(W), m, n, _ld(W, n) if ldw is None else ldw,
                                                 _ptr(abs_sum), _ptr(count), f, _ptr(idx), _ptr(mdiag), _ptr(W_o),
                                                 _ptr(score))


def aser_quantize_rtn(ctx: Context, W, idx, mdiag, f: int, bits: int, layout: int, codes, scales, T=None, *, m=None,
                      n=None, ldw=None, ldt=None) -> int:
    m = W.shape[0] if m is None else m
    n = W.shape[1] if n is None else n
    return ctx._lib.aser_quantize_rtn(ctx.handle, _ptr(W), m, n, _ld(W, n) if ldw is None else ldw, _ptr(idx),
                                      _ptr(mdiag), f, bits, layout, _ptr(codes), _ptr(scales), _ptr(T),
                                      (_ld(T, n) if T is not None else n) if ldt is None else ldt)


def aser_smoothed_weight(ctx: Context, W, idx, f: int, Ws, *, m=None, n=None, ldw=None, ldws=None) -> int:
    m = W.shape[0] if m is None else m
    n = W.shape[1] if n is None else n
    return ctx._lib.aser_smoothed_weight(ctx.handle, _ptr(W), m, n, _ld(W, n) if ldw is None else ldw, _ptr(idx), f,
                                         _ptr(Ws), _ld(Ws, n) if ldws is None else ldws)


def aser_quant_target(ctx: Context, W, mdiag, Wq, T, *, m=None, n=None, ldw=None, ldq=None, ldt=None) -> int:
    m = W.shape[0] if m is None else m
    n = W.shape[1] if n is None else n
    return ctx._lib.aser_quant_target(ctx.handle, _ptr(W), m, n, _ld(W, n) if ldw is None else ldw, _ptr(mdiag),
                                      _ptr(Wq), _ld(Wq, n) if ldq is None else ldq, _ptr(T),
                                      _ld(T, n) if ldt is None else ldt)


def aser_whiten(ctx: Context, G, mdiag, damp: float, S, *, n=None, ldg=None, lds=None, want_info: bool = True):
    """Returns (status, info).  want_info=False passes info = NULL: no synchronisation, a non-positive
    pivot is reported by the next aser_error_reconstruct on this context (info is returned as None)."""
    n = G.shape[0] if n is None else n
    info = ctypes.c_int32(0)
    st = ctx._lib.aser_whiten(ctx.handle, _ptr(G), _ld(G, n) if ldg is None else ldg, n, _ptr(mdiag), float(damp),
                              _ptr(S), _ld(S, n) if lds is None else lds, ctypes.byref(info) if want_info else None)
    return st, (info.value if want_info else None)


def aser_error_reconstruct(ctx: Context, T, S, r: int, L_A, L_B, sigma, opts: Optional[aser_svd_opts] = None, *,
                           idx=None, f: int = 0, m=None, n=None, ldt=None, lds=None):
    """Returns (status, err, n_iter).  idx, f: the outlier set of aser_smooth_outliers (f = 0: none)."""
    m = T.shape[0] if m is None else m
    n = T.shape[1] if n is None else n
    err = ctypes.c_double(0.0)
    nit = ctypes.c_int32(0)
    st = ctx._lib.aser_error_reconstruct(ctx.handle, _ptr(T), m, n, _ld(T, n) if ldt is None else ldt, _ptr(S),
                                         _ld(S, n) if lds is None else lds, r, _ptr(idx) if f > 0 else None, f,
                                         ctypes.byref(opts) if opts is not None else None, _ptr(L_A), _ptr(L_B),
                                         _ptr(sigma), ctypes.byref(err), ctypes.byref(nit))
    return st, err.value, nit.value


def aser_error_reconstruct_enqueue(ctx: Context, T, S, r: int, L_A, L_B, sigma, opts: Optional[aser_svd_opts] = None, *,
                                   idx=None, f: int = 0, m=None, n=None, ldt=None, lds=None) -> int:
    """aser_error_reconstruct without its wait; aser_finish(ctx) returns the results."""
    m = T.shape[0] if m is None else m
    n = T.shape[1] if n is None else n
    return ctx._lib.aser_error_reconstruct_enqueue(ctx.handle, _ptr(T), m, n, _ld(T, n) if ldt is None else ldt, _ptr(S),
                                                   _ld(S, n) if lds is None else lds, r, _ptr(idx) if f > 0 else None, f,
                                                   ctypes.byref(opts) if opts is not None else None, _ptr(L_A),
                                                   _ptr(L_B), _ptr(sigma))


def aser_finish(ctx: Context):
    """Returns (status, err, n_iter) of the enqueued aser_error_reconstruct."""
    err = ctypes.c_double(0.0)
    nit = ctypes.c_int32(0)
    st = ctx._lib.aser_finish(ctx.handle, ctypes.byref(err), ctypes.byref(nit))
    return st, err.value, nit.value


def aser_svd_plan(m: int, n: int, r: int, opts: Optional[aser_svd_opts] = None):
    """Returns (status, block, iters): what aser_error_reconstruct will use for this shape."""
    b, it = ctypes.c_int32(0), ctypes.c_int32(0)
    st = load_library().aser_svd_plan(m, n, r, ctypes.byref(opts) if opts is not None else None, ctypes.byref(b),
                                      ctypes.byref(it))
    return st, b.value, it.value


def aser_quantize_act_rtn(ctx: Context, X, mdiag, bits: int, codes, scales, *, rows=None, n=None, ldx=None,
                          x_dtype=None) -> int:
    rows = X.shape[0] if rows is None else rows
    n = X.shape[1] if n is None else n
    return ctx._lib.aser_quantize_act_rtn(ctx.handle, _ptr(X), _dtype_code(X) if x_dtype is None else x_dtype, rows, n,
                                          _ld(X, n) if ldx is None else ldx, _ptr(mdiag), bits, _ptr(codes),
                                          _ptr(scales))


def aser_spectrum_workspace_bytes(m: int, n: int, with_s: bool) -> int:
    return int(load_library().aser_spectrum_workspace_bytes(m, n, 1 if with_s else 0))


def aser_singular_values(ctx: Context, T, S, sigma, *, m=None, n=None, ldt=None, lds=None) -> int:
    m = T.shape[0] if m is None else m
    n = T.shape[1] if n is None else n
    return ctx._lib.aser_singular_values(ctx.handle, _ptr(T), m, n, _ld(T, n) if ldt is None else ldt, _ptr(S),
                                         (_ld(S, n) if S is not None else n) if lds is None else lds, _ptr(sigma))


def aser_select_rank(ctx: Context, sigma, alpha: float, *, k=None):
    """Returns (status, r, (sum, share_at_r, share_at_r_plus_1))."""
    k = sigma.shape[0] if k is None else k
    r = ctypes.c_int32(0)
    st3 = (ctypes.c_double * 3)()
    st = ctx._lib.aser_select_rank(ctx.handle, _ptr(sigma), k, float(alpha), ctypes.byref(r), st3)
    return st, r.value, (st3[0], st3[1], st3[2])


def aser_effective_rank(ctx: Context, sigma, eps: float = 1e-12, *, k=None):
    """Returns (status, effective_rank)."""
    k = sigma.shape[0] if k is None else k
    out = ctypes.c_double(0.0)
    st = ctx._lib.aser_effective_rank(ctx.handle, _ptr(sigma), k, float(eps), ctypes.byref(out))
    return st, out.value


def aser_output_error_workspace_bytes(m: int, n: int, rows: int, r: int) -> int:
    return int(load_library().aser_output_error_workspace_bytes(m, n, rows, r))


def aser_layer_output_error(ctx: Context, W, X, mdiag, codes, layout: int, scales, L_A, L_B, r: int, act_bits: int, *,
                            m=None, n=None, ldw=None, rows=None, ldx=None, x_dtype=None):
    """Returns (status, err, ref_norm)."""
    m = W.shape[0] if m is None else m
    n = W.shape[1] if n is None else n
    rows = X.shape[0] if rows is None else rows
    err, ref = ctypes.c_double(0.0), ctypes.c_double(0.0)
    st = ctx._lib.aser_layer_output_error(ctx.handle, _ptr(W), m, n, _ld(W, n) if ldw is None else ldw, _ptr(X),
                                          _dtype_code(X) if x_dtype is None else x_dtype, rows,
                                          _ld(X, n) if ldx is None else ldx, _ptr(mdiag), _ptr(codes), layout,
                                          _ptr(scales), _ptr(L_A), _ptr(L_B), r, act_bits, ctypes.byref(err),
                                          ctypes.byref(ref))
    return st, err.value, ref.value


def aser_forward_workspace_bytes(rows: int, n: int, m: int, r: int) -> int:
    return int(load_library().aser_forward_workspace_bytes(rows, n, m, r))


def aser_compensated_forward(ctx: Context, x_codes, x_scales, w_codes, layout: int, w_scales, L_A, L_B, r: int,
                             lowrank_split: bool, Y, *, rows=None, n=None, m=None, ldy=None) -> int:
    rows = x_codes.shape[0] if rows is None else rows
    n = x_codes.shape[1] if n is None else n
    m = w_scales.shape[0] if m is None else m
    return ctx._lib.aser_compensated_forward(ctx.handle, _ptr(x_codes), _ptr(x_scales), rows, n, _ptr(w_codes), layout,
                                             _ptr(w_scales), m, _ptr(L_A), _ptr(L_B), r, 1 if lowrank_split else 0,
                                             _ptr(Y), _ld(Y, m) if ldy is None else ldy)


# ----------------------------------------------------------------------------------- serving
class KvCache:
    """A paged cache of keys and values from its tensors: k, v of pages x key/value heads x slots x channels (bfloat16 or
    int8; any strides that the C struct allows, the same for both), and for int8 the scales, pages x heads x slots fp32."""

    def __init__(self, k, v, k_scale=None, v_scale=None):
        import torch
        if k.shape != v.shape or k.stride() != v.stride() or k.dtype != v.dtype or k.dim() != 4 or k.stride(3) != 1:
            raise ValueError("k and v must be alike, pages x heads x slots x channels with unit channel stride")
        if k.dtype not in (torch.bfloat16, torch.int8):
            raise TypeError("a cache holds bfloat16 or int8")
        if (k.dtype == torch.int8) != (k_scale is not None and v_scale is not None):
            raise ValueError("an int8 cache has scales, a bfloat16 cache has none")
        for sc in (k_scale, v_scale):
            if sc is not None and (sc.dtype != torch.float32 or tuple(sc.shape) != tuple(k.shape[:3]) or not sc.is_contiguous()):
                raise ValueError("scales must be contiguous float32, pages x heads x slots")
        self.device = _same_device(k, v, k_scale, v_scale)
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.c = aser_kv_cache(_ptr(k), _ptr(v), _ptr(k_scale), _ptr(v_scale), k.shape[0], k.stride(0), k.stride(1), k.stride(2),
                               ASER_KV_INT8 if k.dtype == torch.int8 else ASER_KV_BF16, k.shape[2], k.shape[1], k.shape[3])
        self.ref, self.head_dim, self.kv_width, self.page_size = ctypes.byref(self.c), k.shape[3], k.shape[1] * k.shape[3], k.shape[2]

    @classmethod
    def empty(cls, n_pages: int, n_kv: int, page_size: int, head_dim: int, int8: bool = False, device: int = 0):
        """A zeroed cache, pages x heads x slots x channels."""
        import torch
        dev, shape = "cuda:%d" % device, (n_pages, n_kv, page_size, head_dim)
        k, v = (torch.zeros(shape, dtype=torch.int8 if int8 else torch.bfloat16, device=dev) for _ in range(2))
        scales = [torch.zeros(shape[:3], dtype=torch.float32, device=dev) for _ in range(2)] if int8 else [None, None]
        return cls(k, v, *scales)


class KvBatch:
    """The requests of a batch (C struct aser_kv_batch) from its device tensors: start (n_seq + 1), kv_len (n_seq) and the page
    table (n_seq x columns), int32.  Their contents may change between calls; tokens, max_new and max_kv bound them."""

    def __init__(self, start, kv_len, pages, *, tokens: int, max_new: int, max_kv: int):
        import torch
        n_seq = kv_len.shape[0]
        if start.shape[0] != n_seq + 1 or pages.dim() != 2 or pages.shape[0] != n_seq:
            raise ValueError("start has n_seq + 1 entries, kv_len n_seq, pages n_seq rows")
        if any(t.dtype != torch.int32 for t in (start, kv_len, pages)) or not (start.is_contiguous() and kv_len.is_contiguous()):
            raise TypeError("start, kv_len and pages must be int32, start and kv_len contiguous")
        if pages.shape[1] > 1 and pages.stride(1) != 1:
            raise ValueError("the page table must have unit column stride")
        self.device = _same_device(start, kv_len, pages)
        self.start, self.kv_len, self.pages = start, kv_len, pages
        ld = pages.stride(0) if n_seq > 1 else pages.shape[1]
        self.c = aser_kv_batch(_ptr(start), _ptr(kv_len), _ptr(pages), ld, tokens, n_seq, max_new, max_kv)
        self.ref, self.tokens, self.columns, self.max_kv = ctypes.byref(self.c), tokens, pages.shape[1], max_kv


def _refuse(device: int, cache: KvCache, batch: KvBatch):
    if cache.device != device or batch.device != device:
        raise ValueError(_ELSEWHERE)
    raise ValueError("the page table must have a column for every page of max_kv tokens")


_ELSEWHERE = "every tensor must be on the context's device"


def _same_device(*tensors) -> int:
    devices = {t.get_device() for t in tensors if t is not None}
    if len(devices) != 1:
        raise ValueError("the tensors must be on one device")
    return devices.pop()


def _rows(t, rows: int, dtype, device: int):
    """(address, leading dimension, columns) of a matrix of at least `rows` rows.  A kernel that follows an address on another device faults."""
    have, cols = t.shape
    ld, unit = t.stride()
    if have < rows or unit != 1:
        raise ValueError("matrices need a row for each token and unit column stride")
    if t.dtype != dtype:
        raise TypeError("%s expected, got %s" % (dtype, t.dtype))
    if t.get_device() != device:
        raise ValueError(_ELSEWHERE)
    return t.data_ptr(), ld, cols


def _floats(tensors, f32, device: int) -> list:
    """Addresses of dense float32 tensors, None where one is None."""
    found = []
    for t in tensors:
        if t is None:
            found.append(None)
            continue
        if t.dtype != f32:
            raise TypeError("tables, weights and scales must be float32")
        if not t.is_contiguous():
            raise ValueError("tables, weights and scales must be contiguous")
        if t.get_device() != device:
            raise ValueError(_ELSEWHERE)
        found.append(t.data_ptr())
    return found


def aser_kv_append(ctx: Context, q, k, v, cache: KvCache, batch: KvBatch, q_out, *, rope_cos=None, rope_sin=None, interleaved: bool = False,
                   q_norm=None, k_norm=None, eps: float = 1e-6) -> int:
    """q, k, v: tokens x (heads * channels), bfloat16 or float32 alike (q and q_out may be None); rope_cos, rope_sin: positions x
    (rotated channels / 2) float32; q_norm, k_norm: channels of a head, float32."""
    bf16, f32, _ = _TYPES or _types()
    dtype, tokens, device, opts = k.dtype, batch.tokens, ctx.device, None
    dt = ASER_DTYPE_F32 if dtype == f32 else _dtype_code(k)
    if cache.device != device or batch.device != device or batch.columns * cache.page_size < batch.max_kv:
        _refuse(device, cache, batch)
    if (rope_cos is None) != (rope_sin is None):
        raise ValueError("rope_cos and rope_sin go together")
    if rope_cos is not None or q_norm is not None or k_norm is not None:
        # the kernel reads n_pos x half floats of the tables and a float for each channel of a head of the weights
        n_pos = half = 0
        if rope_cos is not None:
            n_pos, half = shape = rope_cos.shape
            if rope_sin.shape != shape:
                raise ValueError("rope_cos and rope_sin must be alike")
        if (q_norm is not None and q_norm.numel() != cache.head_dim) or (k_norm is not None and k_norm.numel() != cache.head_dim):
            raise ValueError("q_norm and k_norm must have a weight for each channel of a head")
        opts = ctypes.byref(aser_qk_opts(*_floats((rope_cos, rope_sin, q_norm, k_norm), f32, device), n_pos, 2 * half, 1 if interleaved else 0, eps))
    kp, ldk, k_width = _rows(k, tokens, dtype, device)
    vp, ldv, v_width = _rows(v, tokens, dtype, device)
    if k_width < cache.kv_width or v_width < cache.kv_width:
        raise ValueError("k and v must have the channels of all key/value heads")
    qp = op = None
    ldq = ldo = heads = 0
    if q is not None:
        qp, ldq, width = _rows(q, tokens, dtype, device)
        op, ldo, out_width = _rows(q_out, tokens, bf16, device)
        heads, rest = divmod(width, cache.head_dim)
        if rest or out_width < width:
            raise ValueError("q must have whole heads, q_out must be as wide")
    return ctx._lib.aser_kv_append(ctx.handle, qp, ldq, heads, kp, ldk, vp, ldv, dt, opts, cache.ref, batch.ref, op, ldo)


def aser_paged_attention_workspace_bytes(cache: KvCache, batch: KvBatch, n_heads: int) -> int:
    return int(load_library().aser_paged_attention_workspace_bytes(cache.ref, batch.ref, n_heads))


def aser_paged_attention(ctx: Context, q, cache: KvCache, batch: KvBatch, out, *, scale: float, window: int = 0, sinks: int = 0) -> int:
    """q, out: tokens x (heads * channels), bfloat16."""
    bf16, device, tokens = (_TYPES or _types())[0], ctx.device, batch.tokens
    if cache.device != device or batch.device != device or batch.columns * cache.page_size < batch.max_kv:
        _refuse(device, cache, batch)
    qp, ldq, width = _rows(q, tokens, bf16, device)
    op, ldo, out_width = _rows(out, tokens, bf16, device)
    heads, rest = divmod(width, cache.head_dim)
    if rest or out_width < width:
        raise ValueError("q must have whole heads, out must be as wide")
    return ctx._lib.aser_paged_attention(ctx.handle, qp, ldq, heads, cache.ref, batch.ref, scale, window, sinks, op, ldo)


def aser_adapter_workspace_bytes(rows: int, n: int, m: int, r: int) -> int:
    return int(load_library().aser_adapter_workspace_bytes(rows, n, m, r))


def aser_adapter_forward(ctx: Context, X, adapter, A, B, scale, Y0, Y) -> int:
    """X: rows x n; adapter: rows int32; A: adapters x r x n and B: adapters x m x r, contiguous bfloat16; scale: adapters float32
    or None; Y0 (None: zeros) and Y: rows x m float32."""
    (n_adapters, r, n), (rows, cols), (b_adapters, m, b_r) = A.shape, X.shape, B.shape
    device, (bf16, f32, i32) = ctx.device, _TYPES or _types()
    if cols != n or b_adapters != n_adapters or b_r != r or not (A.is_contiguous() and B.is_contiguous()):
        raise ValueError("A must be adapters x r x n and B adapters x m x r, contiguous")
    if A.dtype != bf16 or B.dtype != bf16 or adapter.dtype != i32:
        raise TypeError("A and B must be bfloat16, adapter int32")
    if A.get_device() != device or B.get_device() != device or adapter.get_device() != device:
        raise ValueError(_ELSEWHERE)
    if adapter.shape[0] != rows or not adapter.is_contiguous() or (scale is not None and scale.shape[0] < n_adapters):
        raise ValueError("adapter has an int32 for each row of X, contiguous, scale a float32 for each adapter")
    dt = _dtype_code(X)
    xp, ldx, _ = _rows(X, rows, X.dtype, device)
    yp, ldy, width = _rows(Y, rows, f32, device)
    y0p, ldy0, width0 = (None, m, m) if Y0 is None else _rows(Y0, rows, f32, device)
    if width < m or width0 < m:
        raise ValueError("Y0 and Y must be as wide as B is high")
    return ctx._lib.aser_adapter_forward(ctx.handle, xp, dt, rows, n, ldx, adapter.data_ptr(), A.data_ptr(), B.data_ptr(),
                                         _floats((scale,), f32, device)[0], n_adapters, r, m, y0p, ldy0, yp, ldy)


# ----------------------------------------------------------------------------------- microscaled 4 bits, experts
class Mx4:
    """Matrices in microscaled 4 bits from their tensors (C struct aser_mx4), uint8 and contiguous, in the library's layout when `rows` is given: codes, panels x
    words x 4 x 16 x 16, and scales, panels x words x 16 x 4, panels being ceil(rows / 16) and words ceil(n / 128); with one more dimension in front
    for several matrices (experts).  Without it codes are rows x 64 words and scales words x rows x 4, and are laid out anew (copies)."""

    def __init__(self, codes, scales, n: int, rows: Optional[int] = None):
        import torch
        words = (n + 127) // 128
        if codes.dtype != torch.uint8 or scales.dtype != torch.uint8:
            raise TypeError("codes and scales must be uint8")
        self.device = _same_device(codes, scales)
        if rows is None:
            if codes.dim() not in (2, 3) or tuple(scales.shape) != tuple(codes.shape[:-2]) + (words, codes.shape[-2], 4) or codes.shape[-1] != 64 * words:
                raise ValueError("codes must be (matrices x) rows x 64 words, scales (matrices x) words x rows x 4")
            rows, pad = codes.shape[-2], -codes.shape[-2] % 16
            codes, scales = codes.unflatten(-1, (words, 4, 16)), scales.transpose(-3, -2)                       # rows first
            if pad:
                codes = torch.nn.functional.pad(codes, (0, 0, 0, 0, 0, 0, 0, pad))
                scales = torch.nn.functional.pad(scales, (0, 0, 0, 0, 0, pad))
            panels = (rows + pad) // 16
            codes = codes.unflatten(-4, (panels, 16)).movedim(-4, -2).contiguous()
            scales = scales.unflatten(-3, (panels, 16)).transpose(-3, -2).contiguous()
        front, panels = tuple(scales.shape[:-4]), (rows + 15) // 16
        if scales.dim() not in (4, 5) or tuple(codes.shape) != front + (panels, words, 4, 16, 16) or tuple(scales.shape) != front + (panels, words, 16, 4):
            raise ValueError("codes must be (matrices x) panels x words x 4 x 16 x 16, scales (matrices x) panels x words x 16 x 4")
        if not (codes.is_contiguous() and scales.is_contiguous()):
            raise ValueError("codes and scales must be contiguous")
        self.codes, self.scales, self.n, self.rows, self.count, self.front = codes, scales, n, rows, front[0] if front else 1, front
        self.c = aser_mx4(_ptr(codes), _ptr(scales), rows, n, self.count)
        self.ref = ctypes.byref(self.c)

    @classmethod
    def empty(cls, rows: int, n: int, count: Optional[int] = None, device: int = 0):
        """Room for one matrix, or with count for several."""
        import torch
        shape = (() if count is None else (count,)) + ((rows + 15) // 16, (n + 127) // 128)
        return cls(*(torch.empty(shape + more, dtype=torch.uint8, device="cuda:%d" % device) for more in ((4, 16, 16), (16, 4))), n, rows)


class ExpertPlan:
    """Which rows go to which experts (C struct aser_expert_plan), from its tensors: ids, order and place, rows x top_k (order and place may be flat), int32,
    weights, rows x top_k float32, offsets, n_experts + 1 int32; all contiguous."""

    def __init__(self, ids, weights, offsets, order, place):
        import torch
        if ids.dim() != 2 or weights.shape != ids.shape or order.numel() != ids.numel() or place.numel() != ids.numel() or offsets.dim() != 1:
            raise ValueError("ids, weights, order and place have rows x top_k entries, offsets n_experts + 1")
        if any(t.dtype != torch.int32 for t in (ids, offsets, order, place)) or weights.dtype != torch.float32:
            raise TypeError("ids, offsets, order and place must be int32, weights float32")
        if not all(t.is_contiguous() for t in (ids, weights, offsets, order, place)):
            raise ValueError("the arrays of a plan must be contiguous")
        self.device = _same_device(ids, weights, offsets, order, place)
        self.ids, self.weights, self.offsets, self.order, self.place = ids, weights, offsets, order, place
        (self.rows, self.top_k), self.n_experts = ids.shape, offsets.shape[0] - 1
        self.positions = self.rows * self.top_k
        self.c = aser_expert_plan(_ptr(ids), _ptr(weights), _ptr(offsets), _ptr(order), _ptr(place), self.rows, self.top_k, self.n_experts)
        self.ref = ctypes.byref(self.c)

    @classmethod
    def empty(cls, rows: int, top_k: int, n_experts: int, device: int = 0):
        import torch
        make = lambda *shape: torch.empty(shape, dtype=torch.int32, device="cuda:%d" % device)             # noqa: E731
        return cls(make(rows, top_k), make(rows, top_k).view(torch.float32), make(n_experts + 1), make(rows * top_k), make(rows * top_k))


def aser_mx4_quantize(ctx: Context, X, out: Mx4, *, mdiag=None, values=None) -> int:
    """X: (matrices x) rows x n, bfloat16 or float32; mdiag: n float32; values: like X (may be X)."""
    device, dtype = ctx.device, X.dtype
    f32 = (_TYPES or _types())[1]
    dt = ASER_DTYPE_F32 if dtype is f32 else _dtype_code(X)
    if X.dim() == 3:
        X = X.view(-1, X.shape[-1])
        values = None if values is None else values.view(-1, values.shape[-1])
    rows, n, mp = X.shape[0], out.n, None
    if out.device != device:
        raise ValueError(_ELSEWHERE)
    xp, ldx, cols = _rows(X, rows, dtype, device)
    if cols != n or rows != out.rows * out.count:
        raise ValueError("X must have the rows and channels of the result")
    if mdiag is not None:
        if mdiag.numel() != n:
            raise ValueError("mdiag must have a float32 for each channel")
        mp = _floats((mdiag,), f32, device)[0]
    vp, ldv, width = (None, n, n) if values is None else _rows(values, rows, dtype, device)
    if width < n:
        raise ValueError("values must be as wide as X")
    return ctx._lib.aser_mx4_quantize(ctx.handle, xp, dt, ldx, mp, out.ref, vp, ldv)


def _product(ctx: Context, x: Mx4, w: Mx4, Y, rows: int, L_A, L_B, swiglu: bool):
    """(address of L_A, of L_B, rank, swiglu, address of Y, its type, its leading dimension) after the checks that the library cannot make."""
    device = ctx.device
    if x.device != device or w.device != device:
        raise ValueError(_ELSEWHERE)
    r, la, lb, outs, dtype = 0, None, None, w.rows, Y.dtype
    bf16, f32, _ = _TYPES or _types()
    if L_A is not None and L_B is not None:
        r = L_A.shape[-1]
        if L_A.shape != w.front + (outs, r) or L_B.shape != w.front + (r, w.n) or not (L_A.is_contiguous() and L_B.is_contiguous()):
            raise ValueError("L_A must be (matrices x) outputs x r and L_B (matrices x) r x channels, contiguous")
        if L_A.dtype is not bf16 or L_B.dtype is not bf16:
            raise TypeError("L_A and L_B must be bfloat16")
        if L_A.get_device() != device or L_B.get_device() != device:
            raise ValueError(_ELSEWHERE)
        if r:
            la, lb = L_A.data_ptr(), L_B.data_ptr()
    elif L_A is not None or L_B is not None:
        raise ValueError("L_A and L_B go together")
    yp, ldy, width = _rows(Y, rows, dtype, device)
    if width < (outs // 2 if swiglu else outs):
        raise ValueError("Y must have a column for each output")
    return la, lb, r, 1 if swiglu else 0, yp, ASER_DTYPE_F32 if dtype is f32 else _dtype_code(Y), ldy


def aser_mx4_forward_workspace_bytes(rows: int, n: int, m: int, r: int) -> int:
    return int(load_library().aser_mx4_forward_workspace_bytes(rows, n, m, r))


def aser_mx4_forward(ctx: Context, x: Mx4, w: Mx4, Y, *, L_A=None, L_B=None, swiglu: bool = False) -> int:
    """Y: rows x outputs (half as many if swiglu), bfloat16 or float32; L_A: outputs x r and L_B: r x channels, contiguous bfloat16."""
    return ctx._lib.aser_mx4_forward(ctx.handle, x.ref, w.ref, *_product(ctx, x, w, Y, x.rows, L_A, L_B, swiglu))


def aser_route_workspace_bytes(rows: int, n_experts: int, top_k: int) -> int:
    return int(load_library().aser_route_workspace_bytes(rows, n_experts, top_k))


@functools.lru_cache(maxsize=64)
def _route_opts(sigmoid, groups, top_groups, group_top, renormalize, scale):
    return ctypes.byref(aser_route_opts(1 if sigmoid else 0, groups, top_groups, group_top, 1 if renormalize else 0, scale))


def aser_route_experts(ctx: Context, logits, plan: ExpertPlan, *, bias=None, sigmoid: bool = False, groups: int = 1, top_groups: int = 1, group_top: int = 1,
                       renormalize: bool = True, scale: float = 1.0) -> int:
    """logits: rows x experts, bfloat16 or float32; bias: experts float32.  Fills the plan."""
    device, f32 = ctx.device, (_TYPES or _types())[1]
    if plan.device != device:
        raise ValueError(_ELSEWHERE)
    lp, ldl, experts = _rows(logits, plan.rows, logits.dtype, device)
    if experts != plan.n_experts or (bias is not None and bias.numel() != experts):
        raise ValueError("logits and bias must have a column for each expert")
    opts = _route_opts(bool(sigmoid), int(groups), int(top_groups), int(group_top), bool(renormalize), float(scale))      # kept by their values
    return ctx._lib.aser_route_experts(ctx.handle, lp, _dtype_code(logits), ldl, None if bias is None else _floats((bias,), f32, device)[0], opts, plan.ref)


def aser_expert_forward_workspace_bytes(positions: int, n: int, m: int, n_experts: int, r: int) -> int:
    return int(load_library().aser_expert_forward_workspace_bytes(positions, n, m, n_experts, r))


def aser_expert_forward(ctx: Context, x: Mx4, w: Mx4, plan: ExpertPlan, Y, *, gather: bool, L_A=None, L_B=None, swiglu: bool = False) -> int:
    """Y: positions x outputs (half as many if swiglu), bfloat16 or float32; L_A: experts x outputs x r and L_B: experts x r x channels, bfloat16."""
    if plan.device != ctx.device:
        raise ValueError(_ELSEWHERE)
    return ctx._lib.aser_expert_forward(ctx.handle, x.ref, w.ref, plan.ref, 1 if gather else 0, *_product(ctx, x, w, Y, plan.positions, L_A, L_B, swiglu))


def aser_expert_combine(ctx: Context, Y, plan: ExpertPlan, out, *, Y0=None) -> int:
    """Y: positions x m, out and Y0 (None: zeros): rows x m, bfloat16 or float32."""
    device = ctx.device
    if plan.device != device:
        raise ValueError(_ELSEWHERE)
    yp, ldy, m = _rows(Y, plan.positions, Y.dtype, device)
    op, ldo, out_width = _rows(out, plan.rows, out.dtype, device)
    y0p, ldy0, width0 = (None, m, m) if Y0 is None else _rows(Y0, plan.rows, out.dtype, device)
    if out_width != m or width0 < m:
        raise ValueError("out and Y0 must be as wide as Y")
    return ctx._lib.aser_expert_combine(ctx.handle, yp, _dtype_code(Y), ldy, m, plan.ref, y0p, ldy0, op, _dtype_code(out), ldo)


# ----------------------------------------------------------------------------------- one layer, end to end
def aser_mfma_rate_probe(ctx: Context, kind: int, workgroups_per_cu: int = 1, iters: int = 20000):
    """(status, 10^12 operations per second) of a pure MFMA loop: kind 0 bf16, kind 1 int8; kinds 2 and 3: the
    same with the operand traffic of a 256 x 256 tile around the instructions (measurement aid)."""
    out = ctypes.c_double(0.0)
    st = ctx._lib.aser_mfma_rate_probe(ctx.handle, int(kind), int(workgroups_per_cu), int(iters), ctypes.byref(out))
    return st, out.value


class LayerBuffers:
    """Device buffers of one layer's calibration state and outputs (allocated with torch)."""

    def __init__(self, m: int, n: int, r: int, f: int, bits: int, packed: bool, device: int = 0,
                 intermediates: bool = True):
        """intermediates=False: no G / abs_sum / count, T and S (aser_calibrate_layers then keeps them in the
        context's workspace while the layer is in flight)."""
        import torch
        dev = "cuda:%d" % device
        self.m, self.n, self.r, self.f, self.bits, self.packed = m, n, r, f, bits, packed
        if not intermediates:
            self._stats = self.G = self.abs_sum = self.count = self.T = self.S = None
            self._outputs(torch, dev)
            return
        # the three statistics share one allocation, so that clearing them is one launch
        g_bytes = (n * n * 4 + 255) // 256 * 256
        a_bytes = (n * 8 + 255) // 256 * 256
        self._stats = torch.zeros(g_bytes + a_bytes + 256, dtype=torch.uint8, device=dev)
        self.G = self._stats[:n * n * 4].view(torch.float32).view(n, n)
        self.abs_sum = self._stats[g_bytes:g_bytes + n * 8].view(torch.float64)
        self.count = self._stats[g_bytes + a_bytes:g_bytes + a_bytes + 8].view(torch.int64)
        self.T = torch.empty((m, n), dtype=torch.float32, device=dev)
        self.S = torch.empty((n, n), dtype=torch.float32, device=dev)
        self._outputs(torch, dev)

    def _outputs(self, torch, dev):
        m, n, r, f, packed = self.m, self.n, self.r, self.f, self.packed
        self.idx = torch.zeros(max(f, 1), dtype=torch.int32, device=dev)
        self.mdiag = torch.empty(n, dtype=torch.float32, device=dev)
        self.codes = torch.empty((m, n // 2 if packed else n), dtype=torch.uint8 if packed else torch.int8, device=dev)
        self.scales = torch.empty(m, dtype=torch.float32, device=dev)
        self.L_A = torch.empty((m, r), dtype=torch.float32, device=dev)
        self.L_B = torch.empty((r, n), dtype=torch.float32, device=dev)
        self.sigma = torch.empty(r, dtype=torch.float32, device=dev)
        self.err = float("nan")

    def reset_statistics(self):
        self._stats.zero_()


def calibrate_layer(ctx: Context, W, X, buf: LayerBuffers, opts: Optional[aser_svd_opts] = None, damp: float = 0.0,
                    accumulate: bool = True):
    """The loop body of Algorithm 1 for one layer: five ABI calls on buffers in `buf`.

    With accumulate=False the Gram statistics already in `buf` are used (layers sharing an input).
    """
    ctx.ensure_workspace(aser_workspace_bytes(buf.m, buf.n, buf.r, opts))
    layout = ASER_CODES_INT4_PACKED if buf.packed else ASER_CODES_INT8
    if accumulate:
        ctx.check(aser_gram_accumulate(ctx, X, buf.G, buf.abs_sum, buf.count))
    ctx.check(aser_smooth_outliers(ctx, W, buf.abs_sum, buf.count, buf.f, buf.idx, buf.mdiag))
    ctx.check(aser_quantize_rtn(ctx, W, buf.idx, buf.mdiag, buf.f, buf.bits, layout, buf.codes, buf.scales, buf.T))
    st, _ = aser_whiten(ctx, buf.G, buf.mdiag, damp, buf.S, want_info=False)   # pivot check at the layer's one sync
    ctx.check(st)
    st, err, _ = aser_error_reconstruct(ctx, buf.T, buf.S, buf.r, buf.L_A, buf.L_B, buf.sigma, opts,
                                        idx=buf.idx, f=buf.f)
    ctx.check(st)
    buf.err = err
    return buf


def layer_desc(W, buf: "LayerBuffers", X=None, clear_stats: bool = False, opts: Optional[aser_svd_opts] = None,
               damp: float = 0.0, stats_from: Optional[int] = None) -> aser_layer_desc:
    """The descriptor of one layer for aser_calibrate_layers from its weight, its buffers and (unless the
    statistics in `buf` are already finished) its activations.  The tensors must outlive the call."""
    d = aser_layer_desc()
    if X is not None:
        d.X, d.x_dtype, d.rows, d.ldx = _ptr(X), _dtype_code(X), X.shape[0], _ld(X, buf.n)
    d.clear_stats = 1 if clear_stats else 0
    d.stats_from = 0 if stats_from is None else stats_from + 1       # index of an earlier layer of the same call
    d.G, d.ldg, d.abs_sum, d.count = _ptr(buf.G), _ld(buf.G, buf.n) if buf.G is not None else 0, _ptr(buf.abs_sum), _ptr(buf.count)
    d.W, d.m, d.n, d.ldw, d.f, d.bits = _ptr(W), buf.m, buf.n, _ld(W, buf.n), buf.f, buf.bits
    d.idx, d.mdiag = _ptr(buf.idx), _ptr(buf.mdiag)
    d.layout = ASER_CODES_INT4_PACKED if buf.packed else ASER_CODES_INT8
    d.r, d.codes, d.scales = buf.r, _ptr(buf.codes), _ptr(buf.scales)
    d.T, d.ldt = _ptr(buf.T), _ld(buf.T, buf.n) if buf.T is not None else 0
    d.damp, d.S, d.lds = damp, _ptr(buf.S), _ld(buf.S, buf.n) if buf.S is not None else 0
    if opts is not None:
        d.opts = ctypes.pointer(opts)
    d.L_A, d.L_B, d.sigma = _ptr(buf.L_A), _ptr(buf.L_B), _ptr(buf.sigma)
    return d


def aser_layer_workspace_bytes(desc: aser_layer_desc) -> int:
    return int(load_library().aser_layer_workspace_bytes(ctypes.byref(desc)))


def aser_calibrate_layers(ctxs, descs) -> int:
    """Runs the layers `descs` (aser_layer_desc) with len(ctxs) of them in flight; per-layer status, err and
    n_iter are left in the descriptors.  Returns the first failing status, or ASER_OK."""
    lib = load_library()
    handles = (ctypes.c_void_p * len(ctxs))(*[c.handle for c in ctxs])
    arr = (aser_layer_desc * len(descs))(*descs)
    st = lib.aser_calibrate_layers(handles, len(ctxs), arr, len(descs))
    for d, a in zip(descs, arr):
        d.err, d.n_iter, d.status = a.err, a.n_iter, a.status
    return st


def aser_pick_concurrent_streams(stream_handles, want: int, device: int = 0):
    """Returns (status, indices): up to `want` of the candidate streams (raw hipStream_t handles) that run
    concurrently with one another."""
    n = len(stream_handles)
    cand = (ctypes.c_void_p * n)(*stream_handles)
    chosen = (ctypes.c_int32 * max(n, 1))()
    cnt = ctypes.c_int32(0)
    st = load_library().aser_pick_concurrent_streams(device, cand, n, want, chosen, ctypes.byref(cnt))
    return st, [chosen[i] for i in range(cnt.value)]
