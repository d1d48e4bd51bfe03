"""ctypes binding of libsparvar.so (argument marshalling only).

Every function here has the name of the C entry point it calls and forwards
torch tensors as raw device pointers, plane strides and the current HIP stream.
No computation happens in Python. If the shared library is missing the first
call raises: there is no fallback path.
"""
from __future__ import annotations

import contextlib
import ctypes
import math
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
# SPARVAR_LIBRARY selects another build of the same library (e.g. the
# host-sanitized one of build_host_sanitized.py); the default is the in-tree build.
LIB_PATH = os.environ.get("SPARVAR_LIBRARY") or os.path.join(_HERE, "libsparvar.so")

OK, ERR_INVALID, ERR_UNSUPPORTED, ERR_CAPACITY, ERR_HIP = 0, -1, -2, -3, -4
BF16, F32 = 0, 1
MAX_SCALES = 32
NOALLOC_MAX_ROWS = 1 << 20  # SPARVAR_NOALLOC_MAX_ROWS

EXPORTS = [
    "sparvar_scale_info",
    "sparvar_dense_attn_fwd",
    "sparvar_select_blocks",
    "sparvar_decision_step",
    "sparvar_cs4a_column_sums",
    "sparvar_cs4a_select_tokens",
    "sparvar_cs4a_row_stride",
    "sparvar_cs4a_map_tokens",
    "sparvar_cs4a_attn_fwd",
    "sparvar_map_index_steps",
    "sparvar_map_index_steps_noalloc",
    "sparvar_kv_compact",
    "sparvar_csla_row_stride",
    "sparvar_csla_block_rows",
    "sparvar_csla_attn_fwd",
    "sparvar_local_blocks_capacity",
    "sparvar_local_blocks",
    "sparvar_map_index_capacity",
    "sparvar_map_index",
    "sparvar_block_sparse_attn_fwd",
    "sparvar_qkv_append",
    "sparvar_kv_quantize",
    "sparvar_kv_dequantize",
    "sparvar_dense_attn_q8_workspace",
    "sparvar_dense_attn_q8_form",
    "sparvar_dense_attn_q8_fwd",
    "sparvar_block_sparse_attn_q8_fwd",
    "sparvar_block_sparse_attn_q8_form",
    "sparvar_kv_quantize_q4",
    "sparvar_kv_dequantize_q4",
    "sparvar_dense_attn_q4_workspace",
    "sparvar_dense_attn_q4_form",
    "sparvar_dense_attn_q4_fwd",
    "sparvar_block_sparse_attn_q4_fwd",
    "sparvar_block_sparse_attn_q4_form",
    "sparvar_key_weights",
    "sparvar_key_weights_ragged",
    "sparvar_key_weights_form",
    "sparvar_kv_evict",
    "sparvar_status_string",
    "sparvar_last_error",
    "sparvar_set_launch_option",
    "sparvar_get_launch_option",
]

# sparvar_launch_option_t, in enum order
LAUNCH_OPTIONS = ["SWIZZLE", "DENSE_WAVES", "DENSE_CHUNK", "DENSE_STAGES", "SPARSE_WAVES", "SPARSE_CHUNK",
                  "SPARSE_STAGES", "SPARSE_GROUP_WAVES", "SPARSE_GROUP_CHUNK", "SPARSE_GROUP_STAGES", "CSLA_CHUNK",
                  "CSLA_STAGES", "CS4A_CHUNK", "DECISION_FUSED"]
OPT_DEFAULT = -(1 << 31)
# sparvar_projection_t
PROJECT_POINT, PROJECT_COVER = 0, 1
PROJECTIONS = {"point": PROJECT_POINT, "cover": PROJECT_COVER, PROJECT_POINT: PROJECT_POINT,
               PROJECT_COVER: PROJECT_COVER}

# sparvar_norm_t, sparvar_rope_layout_t
NORMS = {None: 0, "rms": 1, "l2": 2}
ROPE_LAYOUTS = {"pairs": 0, "halves": 1}


class SparvarError(RuntimeError):
    def __init__(self, status, message):
        super().__init__(f"{message} (status {status})")
        self.status = status


class _CGeometry(ctypes.Structure):
    _fields_ = [
        ("num_scales", ctypes.c_int32),
        ("h", ctypes.POINTER(ctypes.c_int32)),
        ("w", ctypes.POINTER(ctypes.c_int32)),
        ("block_edge", ctypes.c_int32),
        ("num_sink_scales", ctypes.c_int32),
    ]


class _CScaleInfo(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "h", "w", "n_tokens", "token_offset", "n_tokens_le", "tile_h", "tile_w",
        "tiles_h", "tiles_w", "block_offset", "n_blocks_le")]


class _CQ8Cache(ctypes.Structure):
    _fields_ = [
        ("block", ctypes.c_int32),
        ("capacity", ctypes.c_int32),
        ("k", ctypes.c_void_p),
        ("v", ctypes.c_void_p),
        ("bh_stride", ctypes.c_int64),
        ("k_scale", ctypes.c_void_p),
        ("v_scale", ctypes.c_void_p),
        ("scale_bh_stride", ctypes.c_int64),
    ]


class _CQ4Cache(ctypes.Structure):
    _fields_ = [("capacity", ctypes.c_int32), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("bh_stride", ctypes.c_int64),
                ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p), ("scale_bh_stride", ctypes.c_int64)]


class _CNormRope(ctypes.Structure):
    _fields_ = [
        ("norm", ctypes.c_int32),
        ("layout", ctypes.c_int32),
        ("eps", ctypes.c_float),
        ("table_rows", ctypes.c_int32),
        ("q_weight", ctypes.c_void_p),
        ("k_weight", ctypes.c_void_p),
        ("cos_sin", ctypes.c_void_p),
    ]


_lib = None


def load_library(path: str = LIB_PATH):
    """Load libsparvar.so once and declare the C signatures."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with `python -m paper_2602_04361_amd.build`")
    lib = ctypes.CDLL(path)
    i32, i64, f32, vp = ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_void_p
    G = ctypes.POINTER(_CGeometry)
    Q8, NR, Q4 = ctypes.POINTER(_CQ8Cache), ctypes.POINTER(_CNormRope), ctypes.POINTER(_CQ4Cache)
    sig = {
        "sparvar_scale_info": (ctypes.c_int, [G, i32, ctypes.POINTER(_CScaleInfo)]),
        "sparvar_dense_attn_fwd": (ctypes.c_int, [i32, i32, i32, i32, i32, ctypes.c_int, vp, i64, vp, vp, i64, vp,
                                                  vp, f32, vp]),
        "sparvar_select_blocks": (ctypes.c_int, [G, i32, i32, i32, i32, ctypes.c_int, vp, i64, vp, i64, vp, f32, vp,
                                                 vp, i32, vp, vp]),
        "sparvar_decision_step": (ctypes.c_int, [G, i32, i32, i32, i32, ctypes.c_int, vp, i64, vp, vp, i64, vp, vp,
                                                 f32, vp, i32, vp, vp]),
        "sparvar_cs4a_column_sums": (ctypes.c_int, [G, i32, i32, i32, i32, i32, ctypes.c_int, vp, i64, vp, i64, vp,
                                                    f32, vp, vp]),
        "sparvar_cs4a_select_tokens": (ctypes.c_int, [vp, i32, i32, i32, vp, vp]),
        "sparvar_cs4a_row_stride": (i32, [G, i32]),
        "sparvar_map_index_steps": (ctypes.c_int, [G, i32, i32, vp, i32, i32, i32, vp, i32, i32, i32, vp, vp, vp,
                                                   vp, vp]),
        "sparvar_map_index_steps_noalloc": (ctypes.c_int, [G, i32, i32, vp, i32, i32, i32, vp, i32, i32, i32, vp, vp,
                                                           vp, vp, vp]),
        "sparvar_kv_compact": (ctypes.c_int, [G, i32, vp, i32, i32, i32, ctypes.c_int, vp, vp, i64, vp, vp, i64, vp]),
        "sparvar_csla_row_stride": (i32, [G, i32, i32]),
        "sparvar_csla_block_rows": (ctypes.c_int, [G, i32, vp, i32, vp, i32, vp]),
        "sparvar_csla_attn_fwd": (ctypes.c_int, [G, i32, i32, i32, i32, i32, ctypes.c_int, vp, i64, vp, vp, i64, vp,
                                                 vp, ctypes.c_float, vp, i32, vp]),
        "sparvar_cs4a_map_tokens": (ctypes.c_int, [G, i32, i32, i32, i32, i32, i32, vp, vp, i32, vp]),
        "sparvar_cs4a_attn_fwd": (ctypes.c_int, [G, i32, i32, i32, i32, i32, ctypes.c_int, vp, i64, vp, vp, i64, vp,
                                                 vp, f32, vp, i32, i32, vp, i32, vp]),
        "sparvar_local_blocks_capacity": (i64, [G, i32, i32, i32]),
        "sparvar_local_blocks": (ctypes.c_int, [G, i32, i32, i32, vp, vp, i64, vp]),
        "sparvar_map_index_capacity": (i64, [G, i32, i32, i32, i32, i32, i32, i32, i32]),
        "sparvar_map_index": (ctypes.c_int, [G, i32, i32, i32, i32, i32, vp, vp, vp, i32, i32, i32, vp, vp, i64, vp,
                                             vp, vp]),
        "sparvar_block_sparse_attn_fwd": (ctypes.c_int, [G, i32, i32, i32, i32, ctypes.c_int, vp, i64, vp, vp, i64,
                                                         vp, vp, f32, vp, vp, vp, vp]),
        "sparvar_qkv_append": (ctypes.c_int, [i32, i32, i32, i32, ctypes.c_int, i32, i32, vp, i64, i64, vp, vp, i64, i64,
                                              NR, vp, vp, vp, i64, Q8, vp]),
        "sparvar_kv_quantize": (ctypes.c_int, [i32, i32, i32, ctypes.c_int, i32, i32, vp, vp, i64, Q8, vp]),
        "sparvar_kv_dequantize": (ctypes.c_int, [i32, i32, i32, ctypes.c_int, i32, i32, Q8, vp, vp, i64, vp]),
        "sparvar_dense_attn_q8_workspace": (i64, [i32, i32, i32, i32, i32, i32]),
        "sparvar_dense_attn_q8_form": (ctypes.c_int, [i32, i32, i32, i32, i32, i32, i32, ctypes.POINTER(i32)]),
        "sparvar_dense_attn_q8_fwd": (ctypes.c_int, [i32, i32, i32, i32, i32, i32, ctypes.c_int, vp, i64, Q8, vp, vp, vp,
                                                     f32, vp, i64, vp]),
        "sparvar_block_sparse_attn_q8_fwd": (ctypes.c_int, [G, i32, i32, i32, i32, i32, ctypes.c_int, vp, i64, Q8, vp, vp,
                                                            f32, vp, vp, vp, vp]),
        "sparvar_block_sparse_attn_q8_form": (ctypes.c_int, [G, i32, i32, i32, i32, i32, ctypes.POINTER(i32)]),
        "sparvar_kv_quantize_q4": (ctypes.c_int, [i32, i32, i32, ctypes.c_int, i32, i32, vp, vp, i64, Q4, vp]),
        "sparvar_kv_dequantize_q4": (ctypes.c_int, [i32, i32, i32, ctypes.c_int, i32, i32, Q4, vp, vp, i64, vp]),
        "sparvar_dense_attn_q4_workspace": (i64, [i32, i32, i32, i32, i32, i32]),
        "sparvar_dense_attn_q4_form": (ctypes.c_int, [i32, i32, i32, i32, i32, i32, i32, ctypes.POINTER(i32)]),
        "sparvar_dense_attn_q4_fwd": (ctypes.c_int, [i32, i32, i32, i32, i32, i32, ctypes.c_int, vp, i64, Q4, vp, vp, vp,
                                                     f32, vp, i64, vp]),
        "sparvar_block_sparse_attn_q4_fwd": (ctypes.c_int, [G, i32, i32, i32, i32, i32, ctypes.c_int, vp, i64, Q4, vp, vp,
                                                            f32, vp, vp, vp, vp]),
        "sparvar_block_sparse_attn_q4_form": (ctypes.c_int, [G, i32, i32, i32, i32, i32, ctypes.POINTER(i32)]),
        "sparvar_key_weights": (ctypes.c_int, [i32, i32, i32, i32, i32, i32, ctypes.c_int, vp, i64, vp, i64, Q4, vp, vp, vp,
                                               i32, f32, vp, i64, f32, vp]),
        "sparvar_key_weights_ragged": (ctypes.c_int, [i32, i32, i32, i32, i32, i32, ctypes.c_int, vp, i64, vp, i64, Q4, vp, vp,
                                                      vp, i32, vp, f32, vp, i64, f32, vp]),
        "sparvar_key_weights_form": (ctypes.c_int, [i32, i32, i32, i32, i32, i32, ctypes.c_int, ctypes.POINTER(i32)]),
        "sparvar_kv_evict": (ctypes.c_int, [i32, i32, i32, ctypes.c_int, i32, i32, i32, i32, vp, vp, i64, vp, vp, i64, vp,
                                            vp, i64, Q4, Q4, vp, vp, i64, vp]),
        "sparvar_status_string": (ctypes.c_char_p, [ctypes.c_int]),
        "sparvar_last_error": (ctypes.c_char_p, []),
        "sparvar_set_launch_option": (ctypes.c_int, [i32, i32]),
        "sparvar_get_launch_option": (ctypes.c_int, [i32, ctypes.POINTER(ctypes.c_int32)]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    _lib = lib
    return lib


def _check(status):
    if status != OK:
        lib = load_library()
        raise SparvarError(status, lib.sparvar_last_error().decode() or lib.sparvar_status_string(status).decode())


class Geometry:
    """Host-side sparvar_geometry_t: scale sizes, block edge, sink scales."""

    def __init__(self, h, w, block_edge, num_sink_scales):
        self.h = [int(x) for x in h]
        self.w = [int(x) for x in w]
        self.block_edge = int(block_edge)
        self.num_sink_scales = int(num_sink_scales)
        n = len(self.h)
        self._h = (ctypes.c_int32 * n)(*self.h)
        self._w = (ctypes.c_int32 * n)(*self.w)
        self.c = _CGeometry(n, self._h, self._w, self.block_edge, self.num_sink_scales)

    @property
    def ref(self):
        return ctypes.byref(self.c)

    def scale_info(self, l):
        info = _CScaleInfo()
        _check(load_library().sparvar_scale_info(self.ref, int(l), ctypes.byref(info)))
        return {n: getattr(info, n) for n, _ in _CScaleInfo._fields_}


def sparvar_set_launch_option(name, value=None):
    """Set launch option `name` (a LAUNCH_OPTIONS entry) process-wide; None restores its default."""
    _check(load_library().sparvar_set_launch_option(LAUNCH_OPTIONS.index(name),
                                                    OPT_DEFAULT if value is None else int(value)))


def sparvar_get_launch_option(name):
    v = ctypes.c_int32()
    _check(load_library().sparvar_get_launch_option(LAUNCH_OPTIONS.index(name), ctypes.byref(v)))
    return v.value


@contextlib.contextmanager
def launch_options(**opts):
    """Set launch options for the body of a with-statement, then restore the previous values."""
    before = {}
    for n in opts:
        v = sparvar_get_launch_option(n)
        sparvar_set_launch_option(n, None)
        # (a default stays a default: an option set to that value would be taken as asked for)
        before[n] = None if sparvar_get_launch_option(n) == v else v
    try:
        for n, v in opts.items():
            sparvar_set_launch_option(n, v)
        yield
    finally:
        for n, v in before.items():
            sparvar_set_launch_option(n, v)


# ---------------------------------------------------------------- tensor helpers
_torch_module = None


def _torch():
    global _torch_module  # (an import statement takes 0.3 us a call, and a call asks several times)
    if _torch_module is None:
        import torch  # imported lazily so that the geometry helpers work without torch

        _torch_module = torch
    return _torch_module


def _dtype_code(t):
    torch = _torch()
    if t.dtype == torch.bfloat16:
        return BF16
    if t.dtype == torch.float32:
        return F32
    raise SparvarError(ERR_UNSUPPORTED, f"dtype {t.dtype} not supported")


def _plane_stride(t, name):
    """[B,H,rows,d] tensor with d and rows contiguous and evenly spaced planes."""
    stride = t.stride()
    if len(stride) != 4:
        raise SparvarError(ERR_INVALID, f"{name} must be [B,H,rows,d]")
    B, H, _, d = t.shape
    if stride[3] != 1 or stride[2] != d:
        raise SparvarError(ERR_INVALID, f"{name} rows must be contiguous")
    if B > 1 and stride[0] != H * stride[1]:
        raise SparvarError(ERR_INVALID, f"{name} planes must be evenly spaced")
    return stride[1]


def _ptr(t):
    return None if t is None else t.data_ptr()  # (an int: ctypes converts it by the declared argument type)


def _stream(stream):
    # The raw handle of the current stream: building torch's Stream object for it takes
    # 2.6 us, about as long as a launch.
    if stream is not None:
        return stream.cuda_stream
    torch = _torch()
    if torch.cuda.is_initialized():
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return torch.cuda.current_stream().cuda_stream


def _scale(softmax_scale, d):
    return float(1.0 / math.sqrt(d) if softmax_scale is None else softmax_scale)


# ---------------------------------------------------------------- entry points
def sparvar_dense_attn_fwd(q, k, v, o, lse=None, softmax_scale=None, stream=None):
    """O = softmax(scale Q K^T) V over all keys; see sparvar.h."""
    lib = load_library()
    B, H, n_q, d = q.shape
    n_kv = k.shape[2]
    if _plane_stride(v, "v") != _plane_stride(k, "k"):
        raise SparvarError(ERR_INVALID, "k and v must share one plane stride")
    _check(lib.sparvar_dense_attn_fwd(B, H, n_q, n_kv, d, _dtype_code(q), _ptr(q), _plane_stride(q, "q"),
                                      _ptr(k), _ptr(v), _plane_stride(k, "k"), _ptr(o), _ptr(lse),
                                      _scale(softmax_scale, d), _stream(stream)))
    return o, lse


def sparvar_select_blocks(geom, S, q_S, k_leS, lse_S, topk, topk_idx, scores_out=None, scores_in=None,
                          softmax_scale=None, B=None, H=None, d=None, stream=None):
    """Decision-scale pooled scores and per-query-tile top-k; see sparvar.h."""
    lib = load_library()
    if scores_in is None:
        B, H, _, d = q_S.shape
        dt = _dtype_code(q_S)
        qs, ks = _plane_stride(q_S, "q_S"), _plane_stride(k_leS, "k_leS")
    else:
        B, H = scores_in.shape[0], scores_in.shape[1]
        d = 128 if d is None else d
        dt, qs, ks = BF16, 0, 0
    _check(lib.sparvar_select_blocks(geom.ref, S, B, H, d, dt, _ptr(q_S), qs, _ptr(k_leS), ks, _ptr(lse_S),
                                     _scale(softmax_scale, d), _ptr(scores_in), _ptr(scores_out), topk,
                                     _ptr(topk_idx), _stream(stream)))
    return topk_idx


def sparvar_decision_step(geom, S, q_S, k_leS, v_leS, o_S, lse_S, scores_out, topk, topk_idx, softmax_scale=None,
                          stream=None):
    """Dense attention + LSE, pooled scores and top-k at the decision scale; see sparvar.h."""
    lib = load_library()
    B, H, _, d = q_S.shape
    if _plane_stride(v_leS, "v_leS") != _plane_stride(k_leS, "k_leS"):
        raise SparvarError(ERR_INVALID, "k_leS and v_leS must share one plane stride")
    _check(lib.sparvar_decision_step(geom.ref, S, B, H, d, _dtype_code(q_S), _ptr(q_S), _plane_stride(q_S, "q_S"),
                                     _ptr(k_leS), _ptr(v_leS), _plane_stride(k_leS, "k_leS"), _ptr(o_S), _ptr(lse_S),
                                     _scale(softmax_scale, d), _ptr(scores_out), topk, _ptr(topk_idx),
                                     _stream(stream)))
    return topk_idx


def sparvar_cs4a_column_sums(geom, S, C, q_S, k_leS, lse_S, colsum, softmax_scale=None, stream=None):
    """Token column sums over 1-D query blocks of C queries at S; see sparvar.h."""
    lib = load_library()
    B, H, _, d = q_S.shape
    _check(lib.sparvar_cs4a_column_sums(geom.ref, S, C, B, H, d, _dtype_code(q_S), _ptr(q_S), _plane_stride(q_S, "q_S"),
                                        _ptr(k_leS), _plane_stride(k_leS, "k_leS"), _ptr(lse_S),
                                        _scale(softmax_scale, d), _ptr(colsum), _stream(stream)))
    return colsum


def sparvar_cs4a_select_tokens(values, K, inds, stream=None):
    """Top-K per row of values [..., n] into inds [..., K]; see sparvar.h."""
    n = values.shape[-1]
    rows = values.numel() // n
    if not values.is_contiguous() or not inds.is_contiguous() or inds.numel() != rows * K:
        raise SparvarError(ERR_INVALID, "values and inds must be contiguous [rows, n] and [rows, K]")
    _check(load_library().sparvar_cs4a_select_tokens(_ptr(values), rows, n, K, _ptr(inds), _stream(stream)))
    return inds


def sparvar_cs4a_row_stride(geom, K):
    m = load_library().sparvar_cs4a_row_stride(geom.ref, K)
    if m < 0:
        _check(int(m))
    return int(m)


def sparvar_cs4a_map_tokens(geom, S, k, C, B, H, K, inds_S, tokens, M, stream=None):
    """Sink tokens + mapped top-K tokens for every query block of scale k; see sparvar.h."""
    _check(load_library().sparvar_cs4a_map_tokens(geom.ref, S, k, C, B, H, K, _ptr(inds_S), _ptr(tokens), M,
                                                  _stream(stream)))
    return tokens


def sparvar_cs4a_attn_fwd(geom, k, C, q_k, k_lek, v_lek, o, tokens, M, lse=None, mode=0, base=None, base_scale=0,
                          softmax_scale=None, stream=None):
    """Gather attention over token rows (mode 0), O_cache (1) or O_cache upsampled + sparse update (2)."""
    lib = load_library()
    B, H, _, d = q_k.shape
    if _plane_stride(v_lek, "v_lek") != _plane_stride(k_lek, "k_lek"):
        raise SparvarError(ERR_INVALID, "k_lek and v_lek must share one plane stride")
    _check(lib.sparvar_cs4a_attn_fwd(geom.ref, k, C, B, H, d, _dtype_code(q_k), _ptr(q_k), _plane_stride(q_k, "q_k"),
                                     _ptr(k_lek), _ptr(v_lek), _plane_stride(k_lek, "k_lek"), _ptr(o), _ptr(lse),
                                     _scale(softmax_scale, d), _ptr(tokens), M, mode, _ptr(base), base_scale,
                                     _stream(stream)))
    return o


def sparvar_kv_compact(geom, keep, k_src, v_src, k_dst, v_dst, stream=None):
    """Copy the K/V tokens of the kept scales (1-based, ascending) into a compact cache; see sparvar.h."""
    B, H, _, d = k_src.shape
    if _plane_stride(v_src, "v_src") != _plane_stride(k_src, "k_src") or \
            _plane_stride(v_dst, "v_dst") != _plane_stride(k_dst, "k_dst"):
        raise SparvarError(ERR_INVALID, "K and V must share plane strides")
    arr = (ctypes.c_int32 * max(len(keep), 1))(*[int(l) for l in keep])
    _check(load_library().sparvar_kv_compact(geom.ref, len(keep), ctypes.cast(arr, ctypes.c_void_p), B, H, d,
                                             _dtype_code(k_src), _ptr(k_src), _ptr(v_src),
                                             _plane_stride(k_src, "k_src"), _ptr(k_dst), _ptr(v_dst),
                                             _plane_stride(k_dst, "k_dst"), _stream(stream)))
    return k_dst, v_dst


def compact_geometry(geom, keep, num_sink_scales=None):
    """Geometry of the compact cache that keeps scales `keep` (its scales are the kept ones, in order)."""
    keep = [int(l) for l in keep]
    ns = geom.num_sink_scales if num_sink_scales is None else num_sink_scales
    return Geometry([geom.h[l - 1] for l in keep], [geom.w[l - 1] for l in keep], geom.block_edge, ns)


def sparvar_csla_row_stride(geom, k, block):
    m = load_library().sparvar_csla_row_stride(geom.ref, k, block)
    if m < 0:
        _check(int(m))
    return int(m)


def sparvar_csla_block_rows(geom, k, windows, block, rows, stream=None):
    """CSLA key-block rows of every 1-D query block of scale k (windows: one size per scale 1..k); see sparvar.h."""
    win = (ctypes.c_int32 * max(len(windows), 1))(*[int(w) for w in windows])
    if len(windows) != k:
        raise SparvarError(ERR_INVALID, "one window size per scale 1..k is required")
    _check(load_library().sparvar_csla_block_rows(geom.ref, k, ctypes.cast(win, ctypes.c_void_p), block, _ptr(rows),
                                                  rows.shape[-1], _stream(stream)))
    return rows


def sparvar_csla_attn_fwd(geom, k, block, q_k, k_lek, v_lek, o, rows, lse=None, softmax_scale=None, stream=None):
    """Block-sparse attention of scale k over CSLA block rows (shared by every head)."""
    lib = load_library()
    B, H, _, d = q_k.shape
    if _plane_stride(v_lek, "v_lek") != _plane_stride(k_lek, "k_lek"):
        raise SparvarError(ERR_INVALID, "k_lek and v_lek must share one plane stride")
    _check(lib.sparvar_csla_attn_fwd(geom.ref, k, block, B, H, d, _dtype_code(q_k), _ptr(q_k),
                                     _plane_stride(q_k, "q_k"), _ptr(k_lek), _ptr(v_lek), _plane_stride(k_lek, "k_lek"),
                                     _ptr(o), _ptr(lse), _scale(softmax_scale, d), _ptr(rows), rows.shape[-1],
                                     _stream(stream)))
    return o


def sparvar_local_blocks_capacity(geom, k, radius, prev_dilation=0):
    n = load_library().sparvar_local_blocks_capacity(geom.ref, k, radius, prev_dilation)
    if n < 0:
        _check(int(n))
    return int(n)


def sparvar_local_blocks(geom, k, radius, row_ptr, col_idx, prev_dilation=0, stream=None):
    _check(load_library().sparvar_local_blocks(geom.ref, k, radius, prev_dilation, _ptr(row_ptr), _ptr(col_idx),
                                               col_idx.numel(), _stream(stream)))
    return row_ptr, col_idx


def sparvar_map_index_capacity(geom, S, k, B, H, topk, radius, prev_dilation=0, projection=PROJECT_POINT):
    n = load_library().sparvar_map_index_capacity(geom.ref, S, k, B, H, topk, radius, prev_dilation,
                                                  PROJECTIONS[projection])
    if n < 0:
        _check(int(n))
    return int(n)


def sparvar_map_index(geom, S, k, B, H, topk, topk_idx, local_row_ptr, local_col_idx, radius, row_ptr, col_idx,
                      schedule=None, prev_dilation=0, status=None, projection=PROJECT_POINT, stream=None):
    """Mapped + local blocks -> CSR; local_row_ptr/local_col_idx may both be None. status (optional one-element
    int32 device tensor, cleared by the caller) receives ERR_CAPACITY if a supplied local row was cut."""
    _check(load_library().sparvar_map_index(geom.ref, S, k, B, H, topk, _ptr(topk_idx), _ptr(local_row_ptr),
                                            _ptr(local_col_idx), radius, prev_dilation, PROJECTIONS[projection],
                                            _ptr(row_ptr),
                                            _ptr(col_idx), col_idx.numel(), _ptr(schedule), _ptr(status),
                                            _stream(stream)))
    return row_ptr, col_idx, schedule


def sparvar_map_index_steps(geom, S, ks, B, H, topk, topk_idx, radius, row_ptrs, col_idxs, prev_dilation=0,
                            orders=None, projection=PROJECT_POINT, stream=None, noalloc=False):
    """The rows of several target scales in one launch (local rows generated); with orders (one int32 tensor of
    B*H*G_k entries, or None, per step) also the attention launch order of each step. noalloc=True calls
    sparvar_map_index_steps_noalloc (row lengths in the library's fixed scratch; col_idxs need only the row
    slots)."""
    n = len(ks)
    if not (len(row_ptrs) == len(col_idxs) == n):
        raise SparvarError(ERR_INVALID, "one row_ptr and col_idx per step is required")
    k_arr = (ctypes.c_int32 * max(n, 1))(*[int(k) for k in ks])
    rp_arr = (ctypes.c_void_p * max(n, 1))(*[t.data_ptr() for t in row_ptrs])
    ci_arr = (ctypes.c_void_p * max(n, 1))(*[t.data_ptr() for t in col_idxs])
    cap_arr = (ctypes.c_int64 * max(n, 1))(*[t.numel() for t in col_idxs])
    ord_arr = None
    if orders is not None:
        if len(orders) != n:
            raise SparvarError(ERR_INVALID, "one order (or None) per step is required")
        ord_arr = (ctypes.c_void_p * max(n, 1))(*[(t.data_ptr() if t is not None else None) for t in orders])
    lib = load_library()
    fn = lib.sparvar_map_index_steps_noalloc if noalloc else lib.sparvar_map_index_steps
    _check(fn(geom.ref, S, n, k_arr, B, H, topk, _ptr(topk_idx), radius, prev_dilation, PROJECTIONS[projection], rp_arr,
              ci_arr, cap_arr, ord_arr, _stream(stream)))


def sparvar_block_sparse_attn_fwd(geom, k, q_k, k_lek, v_lek, o, row_ptr, col_idx, lse=None, schedule=None,
                                  softmax_scale=None, stream=None):
    """Block-sparse attention of scale-k queries over the kept blocks; see sparvar.h."""
    lib = load_library()
    B, H, _, d = q_k.shape
    if _plane_stride(v_lek, "v_lek") != _plane_stride(k_lek, "k_lek"):
        raise SparvarError(ERR_INVALID, "k_lek and v_lek must share one plane stride")
    _check(lib.sparvar_block_sparse_attn_fwd(geom.ref, k, B, H, d, _dtype_code(q_k), _ptr(q_k),
                                             _plane_stride(q_k, "q_k"), _ptr(k_lek), _ptr(v_lek),
                                             _plane_stride(k_lek, "k_lek"), _ptr(o), _ptr(lse),
                                             _scale(softmax_scale, d), _ptr(row_ptr), _ptr(col_idx),
                                             _ptr(schedule), _stream(stream)))
    return o, lse


# ---------------------------------------------------------------- 8-bit cache
def _whole(name, *values):
    """Numbers that the caller gives, within the 32 bits that the C calls take (ctypes would cut off the rest)."""
    for v in values:
        if not -0x80000000 <= v <= 0x7FFFFFFF:
            raise SparvarError(ERR_INVALID, f"{name}: {v} does not fit 32 bits")


def _here(first, *others):
    """Every tensor is on the current device (None among the others: not given)."""
    dev = first.get_device()
    if dev < 0:
        raise SparvarError(ERR_INVALID, f"a tensor is on {first.device}, not on a GPU")
    if dev != _torch()._C._cuda_getDevice():
        raise SparvarError(ERR_INVALID, f"a tensor is on {first.device}, which is not the current device")
    for t in others:
        if t is not None and t.get_device() != dev:
            raise SparvarError(ERR_INVALID, f"tensors are on {t.device} and {first.device}")
    return dev


def _on(dev, *objects):
    """Caches and maps (or None) whose tensors are on device dev."""
    for x in objects:
        if x is not None and x.device != dev:
            raise SparvarError(ERR_INVALID, f"the tensors of a {type(x).__name__} are on device {x.device}, not on {dev}")


def _shared_device(name, *tensors):
    """The one device that tensors (None: not given) are on; None without any."""
    devices = {t.get_device() for t in tensors if t is not None}
    if len(devices) > 1:
        raise SparvarError(ERR_INVALID, f"the tensors of a {name} are on several devices")
    return devices.pop() if devices else None


def _same(name, t, shape, dtype):
    """t is a contiguous tensor of that shape and dtype."""
    if t.dtype != dtype:
        raise SparvarError(ERR_INVALID, f"{name} is {t.dtype}, {dtype} is required")
    if t.shape != shape or not t.is_contiguous():
        raise SparvarError(ERR_INVALID, f"{name} must be a contiguous {list(shape)} tensor")


def _check_block(block):
    if block not in (16, 32, 64, 128):
        raise SparvarError(ERR_INVALID, f"scale block {block} is not 16, 32, 64 or 128")


class Q8Cache:
    """Host-side sparvar_q8_cache_t over device tensors: codes k, v [B,H_kv,capacity,d] (float8_e4m3fn, or their bytes as
    uint8) and scale bytes k_scale, v_scale [B,H_kv,ceil(capacity / block)] (uint8 or float8_e8m0fnu)."""

    def __init__(self, k, v, k_scale, v_scale, block):
        torch = _torch()
        for name, t, types in (("k", k, (torch.float8_e4m3fn, torch.uint8)), ("v", v, (torch.float8_e4m3fn, torch.uint8)),
                               ("k_scale", k_scale, (torch.uint8, torch.float8_e8m0fnu)),
                               ("v_scale", v_scale, (torch.uint8, torch.float8_e8m0fnu))):
            if t.dtype not in types:
                raise SparvarError(ERR_UNSUPPORTED, f"{name} is {t.dtype}")
        _check_block(block)
        self.bh_stride = _plane_stride(k, "k")
        self.B, self.H_kv, self.capacity, self.d = k.shape
        if k.shape != v.shape or _plane_stride(v, "v") != self.bh_stride:
            raise SparvarError(ERR_INVALID, "k and v must share their shape and plane stride")
        blocks = -(-self.capacity // block)
        for name, t in (("k_scale", k_scale), ("v_scale", v_scale)):
            if t.dim() != 3 or t.shape[:2] != k.shape[:2] or t.shape[2] < blocks or t.stride(2) != 1 or \
                    t.stride(1) != k_scale.stride(1) or (self.B > 1 and t.stride(0) != self.H_kv * t.stride(1)):
                raise SparvarError(ERR_INVALID, f"{name} must be [B,H_kv,>= {blocks}] with evenly spaced planes, as the other's")
        self.block, self.k, self.v, self.k_scale, self.v_scale = int(block), k, v, k_scale, v_scale
        self.device = _shared_device("Q8Cache", k, v, k_scale, v_scale)
        self.planes = (self.B, self.H_kv, self.d)
        self.c = _CQ8Cache(self.block, self.capacity, k.data_ptr(), v.data_ptr(), self.bh_stride, k_scale.data_ptr(),
                           v_scale.data_ptr(), k_scale.stride(1))
        self.ref = ctypes.byref(self.c)

    @classmethod
    def empty(cls, B, H_kv, capacity, d, block=64, device="cuda"):
        """A cache of unwritten tokens."""
        torch = _torch()
        _check_block(block)
        if min(B, H_kv, capacity, d) < 1:
            raise SparvarError(ERR_INVALID, f"a cache of [{B},{H_kv},{capacity},{d}] is empty")
        code = dict(dtype=torch.float8_e4m3fn, device=device)
        scale = dict(dtype=torch.uint8, device=device)
        blocks = -(-capacity // block)
        return cls(torch.empty(B, H_kv, capacity, d, **code), torch.empty(B, H_kv, capacity, d, **code),
                   torch.empty(B, H_kv, blocks, **scale), torch.empty(B, H_kv, blocks, **scale), block)


class NormRope:
    """Host-side sparvar_norm_rope_t: norm None, "rms" or "l2"; fp32 weights [H,d] and [H_kv,d]; cos_sin fp32
    [rows, d/2, 2], a row for each cache token; layout "pairs" (2i, 2i+1) or "halves" (i, i + d/2)."""

    def __init__(self, norm=None, eps=0.0, q_weight=None, k_weight=None, cos_sin=None, layout="pairs"):
        torch = _torch()
        if norm not in NORMS:
            raise SparvarError(ERR_INVALID, f"norm {norm!r} unknown")
        if layout not in ROPE_LAYOUTS:
            raise SparvarError(ERR_INVALID, f"rotation layout {layout!r} unknown")
        for name, t, dim in (("q_weight", q_weight, 2), ("k_weight", k_weight, 2), ("cos_sin", cos_sin, 3)):
            if t is not None and (t.dtype != torch.float32 or t.dim() != dim or not t.is_contiguous()):
                raise SparvarError(ERR_INVALID, f"{name} must be contiguous fp32 with {dim} axes")
        if cos_sin is not None and cos_sin.shape[2] != 2:
            raise SparvarError(ERR_INVALID, "cos_sin must be [rows, d/2, 2]")
        self.q_weight, self.k_weight, self.cos_sin = q_weight, k_weight, cos_sin
        self.norm, self.eps, self.layout = norm, float(eps), layout
        self.device = _shared_device("NormRope", q_weight, k_weight, cos_sin)
        self.q_shape, self.k_shape = (None if t is None else tuple(t.shape) for t in (q_weight, k_weight))
        self.d = None if cos_sin is None else 2 * cos_sin.shape[1]
        self.c = _CNormRope(NORMS[norm], ROPE_LAYOUTS[layout], float(eps), 0 if cos_sin is None else cos_sin.shape[0],
                            _ptr(q_weight), _ptr(k_weight), _ptr(cos_sin))
        self.ref = ctypes.byref(self.c)

    def rows(self, t0, n):
        """The same for a cache whose token 0 is token t0 of this one's table: its rows [t0, t0 + n)."""
        cs = self.cos_sin
        if cs is not None and not 0 <= t0 <= t0 + n <= cs.shape[0]:
            raise SparvarError(ERR_CAPACITY, f"rotation table of {cs.shape[0]} rows has no rows [{t0}, {t0 + n})")
        return NormRope(self.norm, self.eps, self.q_weight, self.k_weight, None if cs is None else cs[t0:t0 + n], self.layout)


def _token_strides(t, name):
    """Batch and token stride of a [B,n,heads,d] tensor whose heads are contiguous."""
    stride = t.stride()
    if len(stride) != 4:
        raise SparvarError(ERR_INVALID, f"{name} must be [B,n,heads,d]")
    B, n, heads, d = t.shape
    if stride[3] != 1 or (stride[2] != d and heads > 1):
        raise SparvarError(ERR_INVALID, f"{name} heads must be contiguous")
    # (an axis of one has no stride of its own; any multiple of 16 bytes will do)
    return stride[0] if B > 1 else 0, stride[1] if n > 1 else heads * d


def sparvar_qkv_append(q, k, v, t0, heads, q_out, k_cache=None, v_cache=None, q8=None, stream=None):
    """Norms, rotation (heads, a NormRope or None) and the append of tokens [t0, t0 + n): queries to q_out [B,H,n,d], keys
    and values to k_cache, v_cache or to an 8-bit cache q8; see sparvar.h."""
    lib = load_library()
    _whole("t0", t0)
    B, n, H, d = q.shape
    kv_shape = k.shape
    H_kv = kv_shape[2]
    qb, qt = _token_strides(q, "q")
    kb, kt = _token_strides(k, "k")
    if v.shape != kv_shape or (v.stride() != k.stride() and _token_strides(v, "v") != (kb, kt)):
        raise SparvarError(ERR_INVALID, "k and v must share their shape and strides")
    if kv_shape != (B, n, H_kv, d):
        raise SparvarError(ERR_INVALID, "q and k must share batch, tokens and d")
    dtype = q.dtype
    dt = _dtype_code(q)
    if k.dtype != dtype or v.dtype != dtype:
        raise SparvarError(ERR_INVALID, "q, k and v must share a dtype")
    _same("q_out", q_out, (B, H, n, d), dtype)
    dev = _here(q, k, v, q_out, k_cache, v_cache)
    if heads is not None:
        if heads.q_shape not in (None, (H, d)) or heads.k_shape not in (None, (H_kv, d)) or heads.d not in (None, d):
            raise SparvarError(ERR_INVALID, f"weights must be [{H},{d}] and [{H_kv},{d}], cos_sin [rows,{d // 2},2]")
        if heads.device is not None:
            _on(dev, heads)
    cs = 0
    if k_cache is not None and v_cache is not None:
        cs = _plane_stride(k_cache, "k_cache")
        if v_cache.shape != k_cache.shape or _plane_stride(v_cache, "v_cache") != cs:
            raise SparvarError(ERR_INVALID, "k_cache and v_cache must share their shape and plane stride")
        if k_cache.dtype != dtype or v_cache.dtype != dtype or k_cache.shape[:2] != (B, H_kv) or k_cache.shape[3] != d:
            raise SparvarError(ERR_INVALID, f"the caches must be [{B},{H_kv},tokens,{d}] of {dtype}")
        if t0 + n > k_cache.shape[2]:
            raise SparvarError(ERR_CAPACITY, f"tokens up to {t0 + n} exceed the cache's {k_cache.shape[2]}")
    if q8 is not None:
        _check_q8(q8, B, H_kv, d, dev)
    _check(lib.sparvar_qkv_append(B, H, H_kv, d, dt, n, t0, _ptr(q), qb, qt, _ptr(k), _ptr(v), kb, kt,
                                  None if heads is None else heads.ref, _ptr(q_out), _ptr(k_cache), _ptr(v_cache), cs,
                                  None if q8 is None else q8.ref, _stream(stream)))
    return q_out


def _check_cache(c, B, H_kv, d, dev):
    if c.planes != (B, H_kv, d):
        raise SparvarError(ERR_INVALID, f"the cache is [{c.B},{c.H_kv},{c.capacity},{c.d}], not of [{B},{H_kv},.,{d}]")
    _on(dev, c)


_check_q8 = _check_cache


def _kv_planes(k, v):
    stride = _plane_stride(k, "k")
    if v.shape != k.shape or v.dtype != k.dtype or _plane_stride(v, "v") != stride:
        raise SparvarError(ERR_INVALID, "k and v must share their shape, dtype and plane stride")
    return stride, _here(k, v)


def sparvar_kv_quantize(k_src, v_src, t0, q8, stream=None):
    """Write rows of k_src, v_src [B,H_kv,n,d] to tokens [t0, t0 + n) of an 8-bit cache; see sparvar.h."""
    lib = load_library()
    _whole("t0", t0)
    B, H_kv, n, d = k_src.shape
    stride, dev = _kv_planes(k_src, v_src)
    _check_q8(q8, B, H_kv, d, dev)
    _check(lib.sparvar_kv_quantize(B, H_kv, d, _dtype_code(k_src), n, t0, _ptr(k_src), _ptr(v_src), stride, q8.ref,
                                   _stream(stream)))
    return q8


def sparvar_kv_dequantize(q8, t0, k_dst, v_dst, stream=None):
    """Read tokens [t0, t0 + n) of an 8-bit cache back to k_dst, v_dst [B,H_kv,n,d]; see sparvar.h."""
    lib = load_library()
    _whole("t0", t0)
    B, H_kv, n, d = k_dst.shape
    stride, dev = _kv_planes(k_dst, v_dst)
    _check_q8(q8, B, H_kv, d, dev)
    _check(lib.sparvar_kv_dequantize(B, H_kv, d, _dtype_code(k_dst), n, t0, q8.ref, _ptr(k_dst), _ptr(v_dst), stride,
                                     _stream(stream)))
    return k_dst, v_dst


def sparvar_dense_attn_q8_workspace(B, H, H_kv, n_q, n_kv, d):
    """Bytes of workspace with which a dense call of these sizes cuts its keys into parts (0: it does not)."""
    _whole("sizes", B, H, H_kv, n_q, n_kv, d)
    n = load_library().sparvar_dense_attn_q8_workspace(B, H, H_kv, n_q, n_kv, d)
    if n < 0:
        _check(int(n))
    return int(n)


def sparvar_dense_attn_q8_form(B, H, H_kv, n_q, n_kv, d, workspace):
    """(waves, sets, parts) that a dense call of these sizes walks with, with a workspace or without; see sparvar.h."""
    _whole("sizes", B, H, H_kv, n_q, n_kv, d)
    form = (ctypes.c_int32 * 3)()
    _check(load_library().sparvar_dense_attn_q8_form(B, H, H_kv, n_q, n_kv, d, int(workspace), form))
    return tuple(form)


def _codes_attn(q, cache, o, lse, *others):
    """The checks that the attention calls over a cache of codes share."""
    shape = q.shape
    dt = _dtype_code(q)
    _same("o", o, shape, q.dtype)
    if lse is not None:
        _same("lse", lse, shape[:3], _torch().float32)
    _check_cache(cache, shape[0], cache.H_kv, shape[3], _here(q, o, lse, *others))
    return dt


def _dense_codes(fn, q, cache, n_kv, o, lse, kv_len, softmax_scale, workspace, stream):
    _whole("n_kv", n_kv)
    B, H, n_q, d = q.shape
    dt = _codes_attn(q, cache, o, lse, kv_len, workspace)
    if kv_len is not None:
        _same("kv_len", kv_len, (B,), _torch().int32)
    size = 0
    if workspace is not None:
        if not workspace.is_contiguous():
            raise SparvarError(ERR_INVALID, "workspace must be contiguous")
        size = workspace.nbytes
    _check(fn(B, H, cache.H_kv, n_q, n_kv, d, dt, _ptr(q), _plane_stride(q, "q"), cache.ref, _ptr(kv_len), _ptr(o), _ptr(lse),
              _scale(softmax_scale, d), _ptr(workspace), size, _stream(stream)))
    return o, lse


def sparvar_dense_attn_q8_fwd(q, q8, n_kv, o, lse=None, kv_len=None, softmax_scale=None, workspace=None, stream=None):
    """Dense attention over the first n_kv tokens (kv_len[b] of them, int32, for entry b) of an 8-bit cache; workspace: a
    contiguous tensor of at least sparvar_dense_attn_q8_workspace() bytes, or None; see sparvar.h."""
    return _dense_codes(load_library().sparvar_dense_attn_q8_fwd, q, q8, n_kv, o, lse, kv_len, softmax_scale, workspace, stream)


def _sparse_codes(fn, geom, k, q_k, cache, o, row_ptr, col_idx, lse, schedule, softmax_scale, stream):
    _whole("k", k)
    B, H, n, d = q_k.shape
    if not 1 <= k <= len(geom.h):
        raise SparvarError(ERR_INVALID, f"scale {k} outside [1, {len(geom.h)}]")
    h, w, e = geom.h[k - 1], geom.w[k - 1], geom.block_edge
    if n != h * w:
        raise SparvarError(ERR_INVALID, f"q_k has {n} rows, scale {k} has {h * w} tokens")
    i32 = _torch().int32
    if row_ptr.dtype != i32 or col_idx.dtype != i32 or (schedule is not None and schedule.dtype != i32):
        raise SparvarError(ERR_INVALID, "row_ptr, col_idx and schedule must be int32")
    # (what row_ptr holds is device data: rows that end past col_idx are the caller's)
    rows = B * H * -(-h // max(1, min(h, e))) * -(-w // max(1, min(w, e)))
    if row_ptr.numel() <= rows or not row_ptr.is_contiguous() or not col_idx.is_contiguous():
        raise SparvarError(ERR_INVALID, f"row_ptr must hold {rows + 1} entries, and it and col_idx must be contiguous")
    if schedule is not None and (schedule.numel() < rows or not schedule.is_contiguous()):
        raise SparvarError(ERR_INVALID, f"schedule must hold {rows} entries and be contiguous")
    dt = _codes_attn(q_k, cache, o, lse, row_ptr, col_idx, schedule)
    _check(fn(geom.ref, k, B, H, cache.H_kv, d, dt, _ptr(q_k), _plane_stride(q_k, "q_k"), cache.ref, _ptr(o), _ptr(lse),
              _scale(softmax_scale, d), _ptr(row_ptr), _ptr(col_idx), _ptr(schedule), _stream(stream)))
    return o, lse


def sparvar_block_sparse_attn_q8_fwd(geom, k, q_k, q8, o, row_ptr, col_idx, lse=None, schedule=None, softmax_scale=None,
                                     stream=None):
    """Block-sparse attention of scale-k queries over the kept blocks of an 8-bit cache; see sparvar.h."""
    return _sparse_codes(load_library().sparvar_block_sparse_attn_q8_fwd, geom, k, q_k, q8, o, row_ptr, col_idx, lse, schedule,
                         softmax_scale, stream)


def sparvar_block_sparse_attn_q8_form(geom, k, B, H, H_kv, d):
    """(waves, parts of a row) that a block-sparse call of these sizes walks with; see sparvar.h."""
    _whole("sizes", k, B, H, H_kv, d)
    form = (ctypes.c_int32 * 2)()
    _check(load_library().sparvar_block_sparse_attn_q8_form(geom.ref, k, B, H, H_kv, d, form))
    return tuple(form)


# ---------------------------------------------------------------- 4-bit cache
class Q4Cache:
    """Host-side sparvar_q4_cache_t over device tensors: packed codes k, v [B,H_kv,capacity,d/2] (uint8, or
    float4_e2m1fn_x2) and scale bytes k_scale, v_scale [B,H_kv,capacity,d/32] (uint8 or float8_e8m0fnu)."""

    def __init__(self, k, v, k_scale, v_scale):
        torch = _torch()
        codes = (torch.uint8, getattr(torch, "float4_e2m1fn_x2", torch.uint8))
        for name, t, types in (("k", k, codes), ("v", v, codes), ("k_scale", k_scale, (torch.uint8, torch.float8_e8m0fnu)),
                               ("v_scale", v_scale, (torch.uint8, torch.float8_e8m0fnu))):
            if t.dtype not in types:
                raise SparvarError(ERR_UNSUPPORTED, f"{name} is {t.dtype}")
        self.bh_stride = _plane_stride(k, "k")
        self.B, self.H_kv, self.capacity, half = k.shape
        self.d = 2 * half
        if self.d not in (64, 128):
            raise SparvarError(ERR_UNSUPPORTED, f"head dim {self.d} not supported (64 or 128)")
        if k.shape != v.shape or _plane_stride(v, "v") != self.bh_stride:
            raise SparvarError(ERR_INVALID, "k and v must share their shape and plane stride")
        scales = (self.B, self.H_kv, self.capacity, self.d // 32)
        for name, t in (("k_scale", k_scale), ("v_scale", v_scale)):
            if t.shape != scales or _plane_stride(t, name) != _plane_stride(k_scale, "k_scale"):
                raise SparvarError(ERR_INVALID, f"{name} must be {list(scales)} with evenly spaced planes, as the other's")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.device = _shared_device("Q4Cache", k, v, k_scale, v_scale)
        self.planes = (self.B, self.H_kv, self.d)
        self.c = _CQ4Cache(self.capacity, k.data_ptr(), v.data_ptr(), self.bh_stride, k_scale.data_ptr(), v_scale.data_ptr(),
                           _plane_stride(k_scale, "k_scale"))
        self.ref = ctypes.byref(self.c)

    @classmethod
    def empty(cls, B, H_kv, capacity, d, device="cuda"):
        """A cache of unwritten tokens."""
        torch = _torch()
        if d not in (64, 128):
            raise SparvarError(ERR_UNSUPPORTED, f"head dim {d} not supported (64 or 128)")
        if min(B, H_kv, capacity) < 1:
            raise SparvarError(ERR_INVALID, f"a cache of [{B},{H_kv},{capacity},{d}] is empty")
        return cls(*(torch.empty(B, H_kv, capacity, n, dtype=torch.uint8, device=device) for n in (d // 2, d // 2, d // 32, d // 32)))


def sparvar_kv_quantize_q4(k_src, v_src, t0, q4, stream=None):
    """Write rows of k_src, v_src [B,H_kv,n,d] to tokens [t0, t0 + n) of a 4-bit cache; see sparvar.h."""
    lib = load_library()
    _whole("t0", t0)
    B, H_kv, n, d = k_src.shape
    stride, dev = _kv_planes(k_src, v_src)
    _check_cache(q4, B, H_kv, d, dev)
    _check(lib.sparvar_kv_quantize_q4(B, H_kv, d, _dtype_code(k_src), n, t0, _ptr(k_src), _ptr(v_src), stride, q4.ref,
                                      _stream(stream)))
    return q4


def sparvar_kv_dequantize_q4(q4, t0, k_dst, v_dst, stream=None):
    """Read tokens [t0, t0 + n) of a 4-bit cache back to k_dst, v_dst [B,H_kv,n,d]; see sparvar.h."""
    lib = load_library()
    _whole("t0", t0)
    B, H_kv, n, d = k_dst.shape
    stride, dev = _kv_planes(k_dst, v_dst)
    _check_cache(q4, B, H_kv, d, dev)
    _check(lib.sparvar_kv_dequantize_q4(B, H_kv, d, _dtype_code(k_dst), n, t0, q4.ref, _ptr(k_dst), _ptr(v_dst), stride,
                                        _stream(stream)))
    return k_dst, v_dst


def sparvar_dense_attn_q4_workspace(B, H, H_kv, n_q, n_kv, d):
    """Bytes of workspace with which a dense call of these sizes cuts its keys into parts (0: it does not)."""
    _whole("sizes", B, H, H_kv, n_q, n_kv, d)
    n = load_library().sparvar_dense_attn_q4_workspace(B, H, H_kv, n_q, n_kv, d)
    if n < 0:
        _check(int(n))
    return int(n)


def sparvar_dense_attn_q4_form(B, H, H_kv, n_q, n_kv, d, workspace):
    """(waves, sets, parts) that a dense call of these sizes walks with, with a workspace or without; see sparvar.h."""
    _whole("sizes", B, H, H_kv, n_q, n_kv, d)
    form = (ctypes.c_int32 * 3)()
    _check(load_library().sparvar_dense_attn_q4_form(B, H, H_kv, n_q, n_kv, d, int(workspace), form))
    return tuple(form)


def sparvar_dense_attn_q4_fwd(q, q4, n_kv, o, lse=None, kv_len=None, softmax_scale=None, workspace=None, stream=None):
    """Dense attention over the first n_kv tokens (kv_len[b] of them, int32, for entry b) of a 4-bit cache; workspace: a
    contiguous tensor of at least sparvar_dense_attn_q4_workspace() bytes, or None; see sparvar.h."""
    return _dense_codes(load_library().sparvar_dense_attn_q4_fwd, q, q4, n_kv, o, lse, kv_len, softmax_scale, workspace, stream)


def sparvar_block_sparse_attn_q4_fwd(geom, k, q_k, q4, o, row_ptr, col_idx, lse=None, schedule=None, softmax_scale=None,
                                     stream=None):
    """Block-sparse attention of scale-k queries over the kept blocks of a 4-bit cache; see sparvar.h."""
    return _sparse_codes(load_library().sparvar_block_sparse_attn_q4_fwd, geom, k, q_k, q4, o, row_ptr, col_idx, lse, schedule,
                         softmax_scale, stream)


def sparvar_block_sparse_attn_q4_form(geom, k, B, H, H_kv, d):
    """(waves, parts of a row) that a block-sparse call of these sizes walks with; see sparvar.h."""
    _whole("sizes", k, B, H, H_kv, d)
    form = (ctypes.c_int32 * 2)()
    _check(load_library().sparvar_block_sparse_attn_q4_form(geom.ref, k, B, H, H_kv, d, form))
    return tuple(form)


# ---------------------------------------------------------------- a cache within a budget
def _weight_planes(name, t, B, H_kv, n):
    """Plane stride of fp32 weights [B,H_kv,>= n] with evenly spaced planes."""
    if t.dtype != _torch().float32:
        raise SparvarError(ERR_INVALID, f"{name} is {t.dtype}, float32 is required")
    shape, stride = t.shape, t.stride()
    if len(shape) != 3 or shape[0] != B or shape[1] != H_kv or shape[2] < n or (stride[2] != 1 and shape[2] > 1):
        raise SparvarError(ERR_INVALID, f"{name} must be [{B},{H_kv},>= {n}] with rows contiguous")
    # (an axis of one has no stride of its own)
    plane = stride[1] if H_kv > 1 else (stride[0] if B > 1 else shape[2])
    if B > 1 and H_kv > 1 and stride[0] != H_kv * plane:
        raise SparvarError(ERR_INVALID, f"{name} planes must be evenly spaced")
    return plane


def _pair(k, v, name):
    """Shape and plane stride of two [B,H,rows,d] tensors that share them and their dtype."""
    shape, stride = k.shape, _plane_stride(k, name)
    if v.shape != shape or v.dtype != k.dtype or (v.stride() != k.stride() and _plane_stride(v, name) != stride):
        raise SparvarError(ERR_INVALID, f"{name}: k and v must share their shape, dtype and plane stride")
    return shape, stride


def sparvar_key_weights(q, n_kv, lse, w, w_old=None, n_old=None, decay=1.0, k_cache=None, q4=None, kv_len=None,
                        softmax_scale=None, stream=None, old_len=None):
    """Attention weight that the first n_kv keys (kv_len[b] of them, int32, for entry b) of k_cache [B,H_kv,tokens,d] or of a
    4-bit cache q4 got from queries q [B,H,n_q,d] with softmax denominators lse: w = decay * w_old + it, w_old counting for
    the first n_old keys (default: all, or none without w_old), of entry b for old_len[b] of them (int32); see sparvar.h."""
    lib = load_library()
    _whole("n_kv", n_kv)
    B, H, n_q, d = q.shape
    dt = _dtype_code(q)
    if n_old is None:
        n_old = 0 if w_old is None else n_kv
    _whole("n_old", n_old)
    _same("lse", lse, (B, H, n_q), _torch().float32)
    dev = _here(q, lse, w, w_old, k_cache, kv_len, old_len)
    if (k_cache is None) == (q4 is None):
        raise SparvarError(ERR_INVALID, "either k_cache or a 4-bit cache is required")
    if q4 is not None:
        _check_cache(q4, B, q4.H_kv, d, dev)
        H_kv, ks = q4.H_kv, 0
    else:
        H_kv, ks = k_cache.shape[1], _plane_stride(k_cache, "k_cache")
        if k_cache.dtype != q.dtype or k_cache.shape[0] != B or k_cache.shape[3] != d:
            raise SparvarError(ERR_INVALID, f"k_cache must be [{B},H_kv,tokens,{d}] of {q.dtype}")
        if n_kv > k_cache.shape[2]:
            raise SparvarError(ERR_CAPACITY, f"{n_kv} keys exceed the cache's {k_cache.shape[2]}")
    if kv_len is not None:
        _same("kv_len", kv_len, (B,), _torch().int32)
    if old_len is not None:
        _same("old_len", old_len, (B,), _torch().int32)
    ws = _weight_planes("w", w, B, H_kv, n_kv)
    if w_old is not None and _weight_planes("w_old", w_old, B, H_kv, n_kv) != ws and B * H_kv > 1:  # (one plane has no stride)
        raise SparvarError(ERR_INVALID, "w and w_old must share their plane stride")
    _check(lib.sparvar_key_weights_ragged(B, H, H_kv, n_q, n_kv, d, dt, _ptr(q), _plane_stride(q, "q"), _ptr(k_cache), ks,
                                          None if q4 is None else q4.ref, _ptr(lse), _ptr(kv_len), _ptr(w_old), n_old,
                                          _ptr(old_len), float(decay), _ptr(w), ws, _scale(softmax_scale, d), _stream(stream)))
    return w


def sparvar_key_weights_form(B, H, H_kv, n_q, n_kv, d, dtype):
    """Keys of a workgroup that such a call takes for queries of `dtype` (0: the form of few queries); see sparvar.h."""
    _whole("sizes", B, H, H_kv, n_q, n_kv, d)
    torch = _torch()
    if dtype not in (torch.bfloat16, torch.float32):
        raise SparvarError(ERR_UNSUPPORTED, f"queries of {dtype}")
    form = (ctypes.c_int32 * 1)()
    _check(load_library().sparvar_key_weights_form(B, H, H_kv, n_q, n_kv, d, BF16 if dtype == torch.bfloat16 else F32, form))
    return form[0]


def sparvar_kv_evict(w, n, n_keep, n_first, n_last, kept, w_out, k_src=None, v_src=None, k_dst=None, v_dst=None, q4_src=None,
                     q4_dst=None, kv_len=None, stream=None):
    """Of the first n tokens (kv_len[b] of them, int32, for entry b) of k_src, v_src [B,H_kv,tokens,d] or of a 4-bit cache,
    move the n_first first, the n_last last and those of largest weight w [B,H_kv,>= n] to rows [0, n_keep) of k_dst, v_dst
    or q4_dst; kept int32 [B,H_kv,n_keep] gets their tokens (-1: none), w_out [B,H_kv,>= n_keep] their weights; see
    sparvar.h."""
    lib = load_library()
    _whole("n, n_keep, n_first, n_last", n, n_keep, n_first, n_last)
    i32 = _torch().int32
    if w.dim() != 3:
        raise SparvarError(ERR_INVALID, "w must be [B,H_kv,tokens]")
    B, H_kv, _ = w.shape
    _same("kept", kept, (B, H_kv, n_keep), i32)
    if kv_len is not None:
        _same("kv_len", kv_len, (B,), i32)
    ws, wo = _weight_planes("w", w, B, H_kv, n), _weight_planes("w_out", w_out, B, H_kv, n_keep)
    if q4_src is None and q4_dst is None:
        if k_src is None or v_src is None or k_dst is None or v_dst is None:
            raise SparvarError(ERR_INVALID, "either k and v or 4-bit caches are required, both ways")
        _here(w, kept, w_out, k_src, v_src, k_dst, v_dst, kv_len)
        (sb, sh, sn, d), ss = _pair(k_src, v_src, "the source")
        (db, dh, dn, dd), ds = _pair(k_dst, v_dst, "the destination")
        dt = _dtype_code(k_src)
        if sb != B or sh != H_kv or db != B or dh != H_kv or dd != d or k_dst.dtype != k_src.dtype:
            raise SparvarError(ERR_INVALID, f"source and destination must be [{B},{H_kv},tokens,{d}] of {k_src.dtype}")
        if n > sn or n_keep > dn:
            raise SparvarError(ERR_CAPACITY, f"{n} tokens of {sn}, {n_keep} kept of {dn}")
    else:
        if q4_src is None or q4_dst is None or not (k_src is None and v_src is None and k_dst is None and v_dst is None):
            raise SparvarError(ERR_INVALID, "either k and v or 4-bit caches are required, both ways")
        dev = _here(w, kept, w_out, kv_len)
        d, dt, ss, ds = q4_src.d, BF16, 0, 0
        _check_cache(q4_src, B, H_kv, d, dev)
        _check_cache(q4_dst, B, H_kv, d, dev)
    _check(lib.sparvar_kv_evict(B, H_kv, d, dt, n, n_keep, n_first, n_last, _ptr(kv_len), _ptr(w), ws, _ptr(k_src),
                                _ptr(v_src), ss, _ptr(k_dst), _ptr(v_dst), ds, None if q4_src is None else q4_src.ref,
                                None if q4_dst is None else q4_dst.ref, _ptr(kept), _ptr(w_out), wo, _stream(stream)))
    return kept
