"""Thin ctypes binding of libcarnator.so: same names as the C ABI, argument marshalling only.

Every step of the path runs in the library's CUDA kernels.  PyTorch is used here for device
memory (tensors passed in, outputs and workspaces allocated) and for the current stream.
The library is loaded on first use; a missing or unloadable library raises -- there is no
fallback of any kind.
"""
from __future__ import annotations

import ctypes
import functools
import math
import os
from typing import NamedTuple, Optional

_PKG_DIR = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG_DIR, "libcarnator.so")

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_CUDA, ERR_DEVICE_TIMEOUT, ERR_DEVICE_CHECK = range(7)
IMPL_AUTO, IMPL_PORTABLE, IMPL_TCGEN05 = 0, 1, 2
MODE_TOPK, MODE_CUMMASS = 0, 1

# every symbol include/carnator.h declares
EXPORTS = [
    "carnator_build_workspace_bytes", "carnator_build_connectivity",
    "carnator_exact_workspace_bytes", "carnator_build_connectivity_exact",
    "carnator_attn_workspace_bytes", "carnator_compact_mask", "carnator_sparse_attn_compacted",
    "carnator_sparse_attn", "carnator_compacted_tiles",
    "carnator_attn_host_arena_bytes", "carnator_sparse_attn_host",
    "carnator_build_host_arena_bytes", "carnator_build_connectivity_host",
    "carnator_sparse_attn_static", "carnator_static_status",
    "carnator_regions_workspace_bytes", "carnator_build_regions", "carnator_fuse_latents",
    "carnator_region_block_flags", "carnator_sparse_attn_region",
    "carnator_seed_workspace_bytes", "carnator_seed_expansion",
    "carnator_layer_norm", "carnator_layer_norm_backward_workspace_bytes", "carnator_layer_norm_backward",
    "carnator_linear_workspace_bytes", "carnator_linear", "carnator_linear_backward_workspace_bytes", "carnator_linear_backward",
    "carnator_rope_frequencies", "carnator_rope",
    "carnator_block_norm", "carnator_block_norm_backward_workspace_bytes", "carnator_block_norm_backward",
    "carnator_quantize_fp8", "carnator_linear_fp8_workspace_bytes", "carnator_linear_fp8",
    "carnator_delta_e00", "carnator_context_discrepancy", "carnator_size_discrepancy", "carnator_shape_discrepancy",
    "carnator_compatibility_gate", "carnator_clopper_pearson_upper",
    "carnator_query_status", "carnator_selftest_wait_timeout", "carnator_debug_set_builder_path", "carnator_status_string", "carnator_last_cuda_error",
    "carnator_kernel_launches", "carnator_version",
]


class Shape(ctypes.Structure):
    """Mirror of carnator_shape."""
    _fields_ = [
        ("B", ctypes.c_int32), ("H", ctypes.c_int32), ("N", ctypes.c_int32), ("D", ctypes.c_int32),
        ("n_text", ctypes.c_int32), ("T", ctypes.c_int32), ("Hg", ctypes.c_int32), ("Wg", ctypes.c_int32),
        ("block_q", ctypes.c_int32), ("block_k", ctypes.c_int32),
        ("q_stride", ctypes.c_int64 * 3), ("k_stride", ctypes.c_int64 * 3),
        ("v_stride", ctypes.c_int64 * 3), ("o_stride", ctypes.c_int64 * 3),
        ("softmax_scale", ctypes.c_float), ("attn_impl", ctypes.c_int32),
    ]

    @property
    def nqb(self) -> int:
        return -(-self.N // self.block_q)

    @property
    def nkb(self) -> int:
        return -(-self.N // self.block_k)


class BuildParams(ctypes.Structure):
    """Mirror of carnator_build_params."""
    _fields_ = [
        ("mode", ctypes.c_int32), ("keep_ratio", ctypes.c_float), ("mass", ctypes.c_float),
        ("window_frames", ctypes.c_int32), ("text_dense", ctypes.c_int32),
        ("count_includes_forced", ctypes.c_int32),
    ]


class NormShape(ctypes.Structure):
    """Mirror of carnator_norm_shape."""
    _fields_ = [
        ("B", ctypes.c_int32), ("H", ctypes.c_int32), ("N", ctypes.c_int32), ("C", ctypes.c_int32),
        ("x_stride", ctypes.c_int64 * 3), ("y_stride", ctypes.c_int64 * 3),
        ("dy_stride", ctypes.c_int64 * 3), ("dx_stride", ctypes.c_int64 * 3),
        ("shift_stride", ctypes.c_int64), ("scale_stride", ctypes.c_int64),
        ("x_dtype", ctypes.c_int32), ("y_dtype", ctypes.c_int32), ("weight_dtype", ctypes.c_int32), ("mod_dtype", ctypes.c_int32),
        ("eps", ctypes.c_float),
    ]


class LinearShape(ctypes.Structure):
    """Mirror of carnator_linear_shape."""
    _fields_ = [
        ("B", ctypes.c_int32), ("N", ctypes.c_int32), ("in_features", ctypes.c_int32), ("out_features", ctypes.c_int32),
        ("x_stride", ctypes.c_int64 * 2), ("y_stride", ctypes.c_int64 * 2),
        ("residual_stride", ctypes.c_int64 * 2), ("z_stride", ctypes.c_int64 * 2), ("dx_stride", ctypes.c_int64 * 2),
        ("w_stride", ctypes.c_int64), ("dw_stride", ctypes.c_int64), ("gate_stride", ctypes.c_int64),
        ("activation", ctypes.c_int32),
        ("y_dtype", ctypes.c_int32), ("bias_dtype", ctypes.c_int32), ("gate_dtype", ctypes.c_int32),
    ]


class RopeShape(ctypes.Structure):
    """Mirror of carnator_rope_shape."""
    _fields_ = [
        ("B", ctypes.c_int32), ("H", ctypes.c_int32), ("N", ctypes.c_int32), ("D", ctypes.c_int32),
        ("n_text", ctypes.c_int32), ("T", ctypes.c_int32), ("Hg", ctypes.c_int32), ("Wg", ctypes.c_int32),
        ("pairs", ctypes.c_int32 * 3), ("offset", ctypes.c_int32 * 3),
        ("x_stride", ctypes.c_int64 * 3), ("y_stride", ctypes.c_int64 * 3), ("pos_stride", ctypes.c_int64 * 2),
        ("axes", ctypes.c_int32), ("layout", ctypes.c_int32), ("inverse", ctypes.c_int32), ("x_dtype", ctypes.c_int32),
        ("amplitude", ctypes.c_float),
    ]


class RopeScaling(ctypes.Structure):
    """Mirror of carnator_rope_scaling."""
    _fields_ = [
        ("pairs", ctypes.c_int32 * 3), ("mode", ctypes.c_int32), ("theta", ctypes.c_double),
        ("factor", ctypes.c_double * 3), ("original", ctypes.c_double * 3), ("low", ctypes.c_double), ("high", ctypes.c_double),
    ]


class BlockNormShape(ctypes.Structure):
    """Mirror of carnator_block_norm_shape."""
    _fields_ = [
        ("B", ctypes.c_int32), ("N", ctypes.c_int32), ("C", ctypes.c_int32), ("post", ctypes.c_int32), ("pre", ctypes.c_int32),
        ("stream_dtype", ctypes.c_int32), ("x_dtype", ctypes.c_int32), ("y_dtype", ctypes.c_int32), ("weight_dtype", ctypes.c_int32), ("mod_dtype", ctypes.c_int32),
        ("r_stride", ctypes.c_int64 * 2), ("x_stride", ctypes.c_int64 * 2), ("s_stride", ctypes.c_int64 * 2), ("y_stride", ctypes.c_int64 * 2),
        ("ds_stride", ctypes.c_int64 * 2), ("dr_stride", ctypes.c_int64 * 2), ("dx_stride", ctypes.c_int64 * 2),
        ("gate_stride", ctypes.c_int64), ("shift_stride", ctypes.c_int64), ("scale_stride", ctypes.c_int64),
        ("post_eps", ctypes.c_float), ("eps", ctypes.c_float), ("residual_scale", ctypes.c_float),
    ]


class QuantizeShape(ctypes.Structure):
    """Mirror of carnator_quantize_shape."""
    _fields_ = [
        ("B", ctypes.c_int32), ("N", ctypes.c_int32), ("K", ctypes.c_int32), ("block_rows", ctypes.c_int32),
        ("x_stride", ctypes.c_int64 * 2), ("q_stride", ctypes.c_int64 * 2), ("scale_stride", ctypes.c_int64 * 3),
        ("x_dtype", ctypes.c_int32),
    ]


class LinearFp8Shape(ctypes.Structure):
    """Mirror of carnator_linear_fp8_shape."""
    _fields_ = [
        ("B", ctypes.c_int32), ("N", ctypes.c_int32), ("in_features", ctypes.c_int32), ("out_features", ctypes.c_int32),
        ("x_stride", ctypes.c_int64 * 2), ("y_stride", ctypes.c_int64 * 2), ("residual_stride", ctypes.c_int64 * 2),
        ("x_scale_stride", ctypes.c_int64 * 3), ("w_stride", ctypes.c_int64), ("w_scale_stride", ctypes.c_int64 * 2),
        ("gate_stride", ctypes.c_int64),
        ("activation", ctypes.c_int32), ("x_dtype", ctypes.c_int32),
        ("y_dtype", ctypes.c_int32), ("bias_dtype", ctypes.c_int32), ("gate_dtype", ctypes.c_int32),
    ]


class CarnatorError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = f"{where}: {status_string(status)} (status {status})"
        detail = last_cuda_error()
        if detail:
            msg += f" [{detail}]"
        super().__init__(msg)


_lib = None


def lib() -> ctypes.CDLL:
    """Load libcarnator.so (once).  Raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2609_32420_b200.build` "
            "(there is no fallback path)")
    L = ctypes.CDLL(LIB_PATH)
    vp, sz, i64 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int64
    ps, pp = ctypes.POINTER(Shape), ctypes.POINTER(BuildParams)
    L.carnator_build_workspace_bytes.restype = sz
    L.carnator_build_workspace_bytes.argtypes = [ps, pp]
    L.carnator_build_connectivity.restype = ctypes.c_int
    L.carnator_build_connectivity.argtypes = [vp, vp, ps, pp, vp, vp, vp, sz, vp]
    L.carnator_exact_workspace_bytes.restype = sz
    L.carnator_exact_workspace_bytes.argtypes = [ps]
    L.carnator_build_connectivity_exact.restype = ctypes.c_int
    L.carnator_build_connectivity_exact.argtypes = [vp, vp, vp, ps, pp, vp, vp, vp, sz, vp]
    L.carnator_attn_workspace_bytes.restype = sz
    L.carnator_attn_workspace_bytes.argtypes = [ps]
    L.carnator_compact_mask.restype = ctypes.c_int
    L.carnator_compact_mask.argtypes = [vp, vp, ps, vp, sz, vp]
    L.carnator_sparse_attn_compacted.restype = ctypes.c_int
    L.carnator_sparse_attn_compacted.argtypes = [vp, vp, vp, ps, vp, vp, vp, sz, vp]
    L.carnator_sparse_attn.restype = ctypes.c_int
    L.carnator_sparse_attn.argtypes = [vp, vp, vp, vp, vp, ps, vp, vp, vp, sz, vp]
    L.carnator_compacted_tiles.restype = ctypes.c_int
    L.carnator_compacted_tiles.argtypes = [ps, vp, sz, vp, ctypes.POINTER(i64)]
    L.carnator_attn_host_arena_bytes.restype = sz
    L.carnator_attn_host_arena_bytes.argtypes = [ps]
    L.carnator_sparse_attn_host.restype = ctypes.c_int
    L.carnator_sparse_attn_host.argtypes = [vp, vp, vp, vp, vp, ps, vp, vp, vp, sz, vp]
    L.carnator_build_host_arena_bytes.restype = sz
    L.carnator_build_host_arena_bytes.argtypes = [ps, pp]
    L.carnator_build_connectivity_host.restype = ctypes.c_int
    L.carnator_build_connectivity_host.argtypes = [vp, vp, ps, pp, vp, vp, sz, vp]
    L.carnator_sparse_attn_static.restype = ctypes.c_int
    L.carnator_sparse_attn_static.argtypes = [vp, vp, vp, vp, vp, ps, vp, vp, vp]
    L.carnator_static_status.restype = ctypes.c_int
    L.carnator_static_status.argtypes = [vp]
    L.carnator_regions_workspace_bytes.restype = sz
    L.carnator_regions_workspace_bytes.argtypes = [ps]
    L.carnator_build_regions.restype = ctypes.c_int
    L.carnator_build_regions.argtypes = [vp, ps, ctypes.c_int32, ctypes.c_int32, vp, vp, vp, vp, sz, vp]
    L.carnator_fuse_latents.restype = ctypes.c_int
    L.carnator_fuse_latents.argtypes = [vp, vp, vp, i64, i64, ctypes.c_int32, vp, vp]
    L.carnator_region_block_flags.restype = ctypes.c_int
    L.carnator_region_block_flags.argtypes = [vp, ps, ctypes.c_int32, ctypes.c_int32, vp, vp]
    L.carnator_sparse_attn_region.restype = ctypes.c_int
    L.carnator_sparse_attn_region.argtypes = [vp, vp, vp, vp, vp, vp, ps, vp, vp, vp, sz, vp]
    L.carnator_seed_workspace_bytes.restype = sz
    L.carnator_seed_workspace_bytes.argtypes = [ps]
    L.carnator_seed_expansion.restype = ctypes.c_int
    L.carnator_seed_expansion.argtypes = [vp, vp, vp, vp, ctypes.c_int32, ctypes.c_int32, ps, vp, vp, vp, sz, vp]
    pn, pl = ctypes.POINTER(NormShape), ctypes.POINTER(LinearShape)
    L.carnator_layer_norm.restype = ctypes.c_int
    L.carnator_layer_norm.argtypes = [vp, vp, vp, vp, vp, pn, vp, vp, vp, vp]
    L.carnator_layer_norm_backward_workspace_bytes.restype = sz
    L.carnator_layer_norm_backward_workspace_bytes.argtypes = [pn]
    L.carnator_layer_norm_backward.restype = ctypes.c_int
    L.carnator_layer_norm_backward.argtypes = [vp, vp, vp, vp, vp, vp, vp, pn, vp, vp, vp, vp, vp, vp, sz, vp]
    L.carnator_linear_workspace_bytes.restype = sz
    L.carnator_linear_workspace_bytes.argtypes = [pl]
    L.carnator_linear.restype = ctypes.c_int
    L.carnator_linear.argtypes = [vp, vp, vp, vp, vp, pl, vp, vp, vp, sz, vp]
    L.carnator_linear_backward_workspace_bytes.restype = sz
    L.carnator_linear_backward_workspace_bytes.argtypes = [pl]
    L.carnator_linear_backward.restype = ctypes.c_int
    L.carnator_linear_backward.argtypes = [vp, vp, vp, vp, vp, pl, vp, vp, vp, vp, vp, sz, vp]
    dbl, pd = ctypes.c_double, ctypes.POINTER(ctypes.c_double)
    L.carnator_rope_frequencies.restype = ctypes.c_int
    L.carnator_rope_frequencies.argtypes = [ctypes.POINTER(RopeScaling), pd, pd]
    L.carnator_rope.restype = ctypes.c_int
    L.carnator_rope.argtypes = [vp, vp, vp, ctypes.POINTER(RopeShape), vp, vp]
    pb = ctypes.POINTER(BlockNormShape)
    L.carnator_block_norm.restype = ctypes.c_int
    L.carnator_block_norm.argtypes = [vp] * 9 + [pb, vp, vp, vp, vp]
    L.carnator_block_norm_backward_workspace_bytes.restype = sz
    L.carnator_block_norm_backward_workspace_bytes.argtypes = [pb]
    L.carnator_block_norm_backward.restype = ctypes.c_int
    L.carnator_block_norm_backward.argtypes = [vp] * 11 + [pb] + [vp] * 10 + [sz, vp]
    L.carnator_quantize_fp8.restype = ctypes.c_int
    L.carnator_quantize_fp8.argtypes = [vp, ctypes.POINTER(QuantizeShape), vp, vp, vp]
    p8 = ctypes.POINTER(LinearFp8Shape)
    L.carnator_linear_fp8_workspace_bytes.restype = sz
    L.carnator_linear_fp8_workspace_bytes.argtypes = [p8]
    L.carnator_linear_fp8.restype = ctypes.c_int
    L.carnator_linear_fp8.argtypes = [vp, vp, vp, vp, vp, vp, vp, p8, vp, vp, sz, vp]
    L.carnator_delta_e00.restype = dbl
    L.carnator_delta_e00.argtypes = [pd, pd]
    L.carnator_context_discrepancy.restype = dbl
    L.carnator_context_discrepancy.argtypes = [pd, pd, ctypes.c_int32]
    L.carnator_size_discrepancy.restype = dbl
    L.carnator_size_discrepancy.argtypes = [dbl, dbl]
    L.carnator_shape_discrepancy.restype = dbl
    L.carnator_shape_discrepancy.argtypes = [vp, ctypes.c_int32, ctypes.c_int32, vp, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32]
    L.carnator_compatibility_gate.restype = ctypes.c_int32
    L.carnator_compatibility_gate.argtypes = [pd, pd, vp, ctypes.c_int32]
    L.carnator_clopper_pearson_upper.restype = dbl
    L.carnator_clopper_pearson_upper.argtypes = [ctypes.c_int32, ctypes.c_int32, dbl]
    L.carnator_query_status.restype = ctypes.c_int
    L.carnator_query_status.argtypes = [vp, vp]
    L.carnator_selftest_wait_timeout.restype = ctypes.c_int
    L.carnator_selftest_wait_timeout.argtypes = [vp, ctypes.c_uint64, vp]
    L.carnator_debug_set_builder_path.restype = None
    L.carnator_debug_set_builder_path.argtypes = [ctypes.c_int32]
    L.carnator_status_string.restype = ctypes.c_char_p
    L.carnator_status_string.argtypes = [ctypes.c_int]
    L.carnator_last_cuda_error.restype = ctypes.c_char_p
    L.carnator_last_cuda_error.argtypes = []
    L.carnator_kernel_launches.restype = i64
    L.carnator_kernel_launches.argtypes = []
    L.carnator_version.restype = ctypes.c_int32
    L.carnator_version.argtypes = []
    _lib = L
    return L


def status_string(status: int) -> str:
    return lib().carnator_status_string(int(status)).decode()


def last_cuda_error() -> str:
    return lib().carnator_last_cuda_error().decode()


def kernel_launches() -> int:
    return int(lib().carnator_kernel_launches())


def version() -> int:
    return int(lib().carnator_version())


def _check(status: int, where: str):
    if status != OK:
        raise CarnatorError(status, where)


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream(stream=None):
    import torch
    if stream is None:
        if torch.cuda.is_initialized():      # the handle itself: a Stream object costs 4 us, a fifth of a small call
            return ctypes.c_void_p(torch._C._cuda_getCurrentRawStream(torch.cuda.current_device()))
        if not torch.cuda.is_available():
            return ctypes.c_void_p(None)     # argument-validation calls on a machine without a GPU
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


def make_shape(B, H, N, D, n_text, T, Hg, Wg, block_q, block_k, Q=None, K=None, V=None, O=None,
               softmax_scale: float = 0.0, attn_impl: int = IMPL_AUTO) -> Shape:
    """Fill a Shape; strides are taken from the given [B,H,rows,D] tensors (contiguous [B,H,N,D] if absent)."""
    s = Shape()
    s.B, s.H, s.N, s.D = B, H, N, D
    s.n_text, s.T, s.Hg, s.Wg = n_text, T, Hg, Wg
    s.block_q, s.block_k = block_q, block_k
    default = (H * N * D, N * D, D)
    for name, t in (("q_stride", Q), ("k_stride", K), ("v_stride", V), ("o_stride", O)):
        st = default if t is None else tuple(t.stride()[:3])
        if t is not None and t.stride()[3] != 1:
            raise ValueError("head dimension must be contiguous")
        setattr(s, name, (ctypes.c_int64 * 3)(*st))
    s.softmax_scale = softmax_scale
    s.attn_impl = attn_impl
    return s


def shape_of(w, Q=None, K=None, V=None, O=None, attn_impl: int = IMPL_AUTO) -> Shape:
    """Shape of a workload record (any object with B,H,N,D,n_text,T,Hg,Wg,block)."""
    return make_shape(w.B, w.H, w.N, w.D, w.n_text, w.T, w.Hg, w.Wg, w.block, w.block, Q, K, V, O,
                      attn_impl=attn_impl)


def params_of(bp) -> BuildParams:
    p = BuildParams()
    p.mode, p.keep_ratio, p.mass = bp.mode, bp.keep_ratio, bp.mass
    p.window_frames, p.text_dense, p.count_includes_forced = bp.window_frames, bp.text_dense, bp.count_includes_forced
    return p


def _made(make, device, stream):
    """make(), the memory of something that a call makes for itself or hands back.  On a stream of the caller's own the memory is that stream's: what is dropped, by the call or
    later by its caller, goes to that stream's later work only, behind the kernels that still use it.  Results are read on the current stream, too, as a rule: it is recorded."""
    if stream is None or device.type != "cuda":
        return make()
    import torch
    reader = torch.cuda.current_stream()
    with torch.cuda.stream(stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(stream.cuda_stream)):
        t = make()
    t.record_stream(reader)
    return t


def _new_ws(nbytes: int, device, stream=None):
    import torch
    return _made(lambda: torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device), device, stream)


# --------------------------------------------------------------------------------------------
# the calls
# --------------------------------------------------------------------------------------------
def build_workspace_bytes(shape: Shape, params: BuildParams) -> int:
    return int(lib().carnator_build_workspace_bytes(ctypes.byref(shape), ctypes.byref(params)))


def attn_workspace_bytes(shape: Shape) -> int:
    return int(lib().carnator_attn_workspace_bytes(ctypes.byref(shape)))


def build_connectivity(Q, K, shape: Shape, params: BuildParams, mask=None, pooled_scores=None, ws=None, stream=None):
    """carnator_build_connectivity.  Returns (mask uint8 [B,H,nqb,nkb], ws)."""
    import torch
    if mask is None:
        mask = _made(lambda: torch.empty((shape.B, shape.H, shape.nqb, shape.nkb), dtype=torch.uint8, device=Q.device), Q.device, stream)
    if ws is None:
        ws = _new_ws(build_workspace_bytes(shape, params), Q.device, stream)
    st = lib().carnator_build_connectivity(_ptr(Q), _ptr(K), ctypes.byref(shape), ctypes.byref(params), _ptr(mask),
                                           _ptr(pooled_scores), _ptr(ws), ws.numel(), _stream(stream))
    _check(st, "carnator_build_connectivity")
    return mask, ws


def exact_workspace_bytes(shape: Shape) -> int:
    return int(lib().carnator_exact_workspace_bytes(ctypes.byref(shape)))


def build_connectivity_exact(Q, K, LSE, shape: Shape, params: BuildParams, mask=None, block_mass=None, ws=None,
                             stream=None):
    """carnator_build_connectivity_exact.  Returns (mask uint8 [B,H,nqb,nkb], ws)."""
    import torch
    if mask is None:
        mask = _made(lambda: torch.empty((shape.B, shape.H, shape.nqb, shape.nkb), dtype=torch.uint8, device=Q.device), Q.device, stream)
    if ws is None:
        ws = _new_ws(exact_workspace_bytes(shape), Q.device, stream)
    st = lib().carnator_build_connectivity_exact(_ptr(Q), _ptr(K), _ptr(LSE), ctypes.byref(shape), ctypes.byref(params),
                                                 _ptr(mask), _ptr(block_mass), _ptr(ws), ws.numel(), _stream(stream))
    _check(st, "carnator_build_connectivity_exact")
    return mask, ws


def compact_mask(mask, recompute_rows, shape: Shape, ws=None, stream=None):
    if ws is None:
        ws = _new_ws(attn_workspace_bytes(shape), mask.device, stream)
    st = lib().carnator_compact_mask(_ptr(mask), _ptr(recompute_rows), ctypes.byref(shape), _ptr(ws), ws.numel(),
                                     _stream(stream))
    _check(st, "carnator_compact_mask")
    return ws


def _outputs(Q, shape: Shape, O, LSE, stream):
    import torch
    if O is None:
        O = _made(lambda: torch.empty((shape.B, shape.H, shape.N, shape.D), dtype=torch.bfloat16, device=Q.device), Q.device, stream)
        st, D, nd = shape.o_stride, shape.D, shape.N * shape.D      # contiguous
        st[0], st[1], st[2] = shape.H * nd, nd, D
    if LSE is None:
        LSE = _made(lambda: torch.empty((shape.B, shape.H, shape.N), dtype=torch.float32, device=Q.device), Q.device, stream)
    return O, LSE


def sparse_attn_compacted(Q, K, V, shape: Shape, ws, O=None, LSE=None, stream=None):
    O, LSE = _outputs(Q, shape, O, LSE, stream)
    st = lib().carnator_sparse_attn_compacted(_ptr(Q), _ptr(K), _ptr(V), ctypes.byref(shape), _ptr(O), _ptr(LSE),
                                              _ptr(ws), ws.numel(), _stream(stream))
    _check(st, "carnator_sparse_attn_compacted")
    return O, LSE


def sparse_attn(Q, K, V, mask, recompute_rows, shape: Shape, O=None, LSE=None, ws=None, stream=None):
    """carnator_sparse_attn.  Returns (O bf16 [B,H,N,D], LSE fp32 [B,H,N], ws)."""
    O, LSE = _outputs(Q, shape, O, LSE, stream)
    if ws is None:
        ws = _new_ws(attn_workspace_bytes(shape), Q.device, stream)
    st = lib().carnator_sparse_attn(_ptr(Q), _ptr(K), _ptr(V), _ptr(mask), _ptr(recompute_rows), ctypes.byref(shape),
                                    _ptr(O), _ptr(LSE), _ptr(ws), ws.numel(), _stream(stream))
    _check(st, "carnator_sparse_attn")
    return O, LSE, ws


def compacted_tiles(shape: Shape, ws, stream=None) -> int:
    out = ctypes.c_int64(0)
    st = lib().carnator_compacted_tiles(ctypes.byref(shape), _ptr(ws), ws.numel(), _stream(stream), ctypes.byref(out))
    _check(st, "carnator_compacted_tiles")
    return int(out.value)


def query_status(ws, stream=None) -> int:
    return int(lib().carnator_query_status(_ptr(ws), _stream(stream)))


def selftest_wait_timeout(ws, limit_ns: int, stream=None) -> None:
    """carnator_selftest_wait_timeout: a bounded wait on a barrier nothing arms; query_status(ws) reports the time-out."""
    _check(lib().carnator_selftest_wait_timeout(_ptr(ws), int(limit_ns), _stream(stream)), "carnator_selftest_wait_timeout")


# byte offsets inside the 256-byte workspace header (tests of the time-out path write them)
HDR_WAIT_LIMIT_NS, HDR_DEBUG_WITHHOLD = 40, 48

BUILDER_AUTO, BUILDER_THREE_KERNELS, BUILDER_FUSED = 0, 1, 2


def debug_set_builder_path(path: int) -> None:
    """Testing aid: 0 = by size, 1 = the separate kernels, 2 = the fused persistent kernel where the shape allows it."""
    lib().carnator_debug_set_builder_path(int(path))


def attn_host_arena_bytes(shape: Shape) -> int:
    return int(lib().carnator_attn_host_arena_bytes(ctypes.byref(shape)))


def sparse_attn_host(Q, K, V, mask, recompute_rows, shape: Shape, O, LSE, arena, stream=None):
    """carnator_sparse_attn_host: Q..LSE are HOST tensors (pinned), arena is a device buffer."""
    st = lib().carnator_sparse_attn_host(_ptr(Q), _ptr(K), _ptr(V), _ptr(mask), _ptr(recompute_rows),
                                         ctypes.byref(shape), _ptr(O), _ptr(LSE), _ptr(arena), arena.numel(),
                                         _stream(stream))
    _check(st, "carnator_sparse_attn_host")


def build_host_arena_bytes(shape: Shape, params: BuildParams) -> int:
    return int(lib().carnator_build_host_arena_bytes(ctypes.byref(shape), ctypes.byref(params)))


def build_connectivity_host(Q, K, shape: Shape, params: BuildParams, mask, arena, stream=None):
    st = lib().carnator_build_connectivity_host(_ptr(Q), _ptr(K), ctypes.byref(shape), ctypes.byref(params),
                                                _ptr(mask), _ptr(arena), arena.numel(), _stream(stream))
    _check(st, "carnator_build_connectivity_host")


STATIC_SCRATCH_BYTES = 8 << 20


def sparse_attn_static(Q, K, V, mask, recompute_rows, shape: Shape, O, LSE, stream=None):
    """carnator_sparse_attn_static: no workspace argument -- the library's built-in scratch array is used.

    For callers that must not allocate device memory when they call (fixed memory budgets, hosts that own
    the allocator, latency-critical loops).  O and LSE must be passed in; nothing is allocated here either.
    Shapes whose workspace exceeds STATIC_SCRATCH_BYTES raise with CARNATOR_ERR_WORKSPACE.  Calls share the
    one array per device: keep them ordered on the GPU.
    """
    shape.o_stride = (ctypes.c_int64 * 3)(*O.stride()[:3])
    st = lib().carnator_sparse_attn_static(_ptr(Q), _ptr(K), _ptr(V), _ptr(mask), _ptr(recompute_rows),
                                           ctypes.byref(shape), _ptr(O), _ptr(LSE), _stream(stream))
    _check(st, "carnator_sparse_attn_static")


def static_status(stream=None) -> int:
    """carnator_static_status: the device status word of the static-scratch form on the current device (read and cleared)."""
    return int(lib().carnator_static_status(_stream(stream)))


DTYPE_F32, DTYPE_BF16, DTYPE_E4M3 = 0, 1, 2


def build_regions(evidence, shape: Shape, r_active: int = 2, r_context: int = 3, stream=None):
    """carnator_build_regions.  evidence uint8 [T,Hg,Wg] on the device -> (active, context, W)."""
    import torch
    active, context = (_made(lambda: torch.empty_like(evidence), evidence.device, stream) for _ in range(2))
    W = _made(lambda: torch.empty(evidence.shape, dtype=torch.float32, device=evidence.device), evidence.device, stream)
    ws = _new_ws(int(lib().carnator_regions_workspace_bytes(ctypes.byref(shape))), evidence.device, stream)
    st = lib().carnator_build_regions(_ptr(evidence), ctypes.byref(shape), r_active, r_context, _ptr(active), _ptr(context),
                                      _ptr(W), _ptr(ws), ws.numel(), _stream(stream))
    _check(st, "carnator_build_regions")
    return active, context, W


def fuse_latents(z_target, z_hist, W, z_out=None, stream=None):
    """carnator_fuse_latents over [channels, tokens] tensors (fp32 or bf16), W fp32 [tokens]."""
    import torch
    if z_out is None:
        z_out = _made(lambda: torch.empty_like(z_target), z_target.device, stream)
    dtype = DTYPE_F32 if z_target.dtype == torch.float32 else DTYPE_BF16
    channels, tokens = z_target.shape[0], z_target[0].numel()
    st = lib().carnator_fuse_latents(_ptr(z_target), _ptr(z_hist), _ptr(W), channels, tokens, dtype, _ptr(z_out), _stream(stream))
    _check(st, "carnator_fuse_latents")
    return z_out


def region_block_flags(region, shape: Shape, block: int, text_value: int = 1, stream=None):
    import torch
    n = shape.n_text + shape.T * shape.Hg * shape.Wg
    flags = _made(lambda: torch.empty((-(-n // block),), dtype=torch.uint8, device=region.device), region.device, stream)
    st = lib().carnator_region_block_flags(_ptr(region), ctypes.byref(shape), block, text_value, _ptr(flags), _stream(stream))
    _check(st, "carnator_region_block_flags")
    return flags


def sparse_attn_region(Q, K, V, mask, active_q, context_k, shape: Shape, O, LSE, ws=None, stream=None):
    """carnator_sparse_attn_region: O and LSE are updated in place; rows of inactive query blocks stay as they are."""
    if ws is None:
        ws = _new_ws(attn_workspace_bytes(shape), Q.device, stream)
    shape.o_stride = (ctypes.c_int64 * 3)(*O.stride()[:3])
    st = lib().carnator_sparse_attn_region(_ptr(Q), _ptr(K), _ptr(V), _ptr(mask), _ptr(active_q), _ptr(context_k),
                                           ctypes.byref(shape), _ptr(O), _ptr(LSE), _ptr(ws), ws.numel(), _stream(stream))
    _check(st, "carnator_sparse_attn_region")
    return ws


def seed_workspace_bytes(shape: Shape) -> int:
    return int(lib().carnator_seed_workspace_bytes(ctypes.byref(shape)))


def seed_expansion(Q, K, LSE, seeds, n_pos: int, n_neg: int, shape: Shape, per_head=None, stream=None, ws=None,
                   return_ws: bool = False):
    """carnator_seed_expansion.  seeds: int32 device tensor [n_pos + n_neg].  Returns contrast fp32 [B,N]
    (and the workspace, whose header carries the device status, with ``return_ws``)."""
    import torch
    out = _made(lambda: torch.empty((shape.B, shape.N), dtype=torch.float32, device=Q.device), Q.device, stream)
    if ws is None:
        ws = _new_ws(int(lib().carnator_seed_workspace_bytes(ctypes.byref(shape))), Q.device, stream)
    st = lib().carnator_seed_expansion(_ptr(Q), _ptr(K), _ptr(LSE), _ptr(seeds), n_pos, n_neg, ctypes.byref(shape),
                                       _ptr(per_head), _ptr(out), _ptr(ws), ws.numel(), _stream(stream))
    _check(st, "carnator_seed_expansion")
    return (out, ws) if return_ws else out


# ---- around the attention: layer norm, projections, their gradients -----------------------------------
ACT_NONE, ACT_GELU_TANH, ACT_GELU, ACT_SILU = 0, 1, 2, 3


def _dtype_code(t, what: str) -> int:
    import torch
    if t.dtype == torch.float32:
        return DTYPE_F32
    if t.dtype == torch.bfloat16:
        return DTYPE_BF16
    raise ValueError(f"{what} must be float32 or bfloat16, not {t.dtype}")


def _dtype_of(code: int):
    import torch
    return torch.float32 if code == DTYPE_F32 else torch.bfloat16 if code == DTYPE_BF16 else torch.float8_e4m3fn


def _fit(t, what: str, dtype, size, stride, device) -> None:
    """A tensor has to be what the shape record says: type, shape, device, and strides (that of an axis of one entry does not matter)."""
    if t.dtype is dtype and t.shape == size and t.stride() == stride and t.device == device:
        return
    if t.dtype is not dtype:
        raise ValueError(f"{what} is {t.dtype}, the shape record says {dtype}")
    if t.device != device:
        raise ValueError(f"{what} is on {t.device}, not on {device}")
    if t.shape != size:
        raise ValueError(f"{what} has shape {tuple(t.shape)}, not {size}")
    for n, a, b in zip(size, t.stride(), stride):
        if n > 1 and a != b:
            raise ValueError(f"{what} has strides {t.stride()}, the shape record says {stride}")


def _stream_on(device, stream):
    """The stream of a call: the current one unless given.  The kernels run on the current device, so the tensors have to be there; a machine without a
    GPU only checks arguments."""
    import torch
    if device.type != "cuda":
        if torch.cuda.is_available():
            raise ValueError(f"the tensors are on {device}: the kernels read memory of the current device only")
        return _stream(stream)
    current = torch.cuda.current_device()
    if device.index != current:
        raise ValueError(f"the tensors are on {device}, the current device is cuda:{current}")
    return ctypes.c_void_p(torch._C._cuda_getCurrentRawStream(current) if stream is None else stream.cuda_stream)


class _Said:
    """What a record says of the tensors of its call, (type, shape, strides) each, and a copy of it for the library.  Made for each content of a record
    and never changed afterwards, so that records may be copied, changed between calls and shared among threads."""
    __slots__ = ("record", "ref", "x", "y", "dy", "dx", "residual", "z", "w", "dw", "vec", "shift", "scale", "gate", "bias", "stat", "freq", "pos", "q",
                 "x_scale", "w_scale", "r", "s", "ds", "dr")

    def __init__(self, record):
        self.record, self.ref = record, ctypes.byref(record)


@functools.lru_cache(maxsize=1024)
def _norm_said(of: bytes) -> _Said:
    s = NormShape.from_buffer_copy(of)
    said = _Said(s)
    size, x, y, w, m = (s.B, s.H, s.N, s.C), _dtype_of(s.x_dtype), _dtype_of(s.y_dtype), _dtype_of(s.weight_dtype), _dtype_of(s.mod_dtype)
    said.x, said.y = (x, size, (*s.x_stride, 1)), (y, size, (*s.y_stride, 1))
    said.dy, said.dx = (y, size, (*s.dy_stride, 1)), (x, size, (*s.dx_stride, 1))
    said.vec = (w, (s.C,), (1,))
    said.shift, said.scale = (m, (s.B, s.C), (s.shift_stride, 1)), (m, (s.B, s.C), (s.scale_stride, 1))
    said.stat = (_dtype_of(DTYPE_F32), size[:3], (s.H * s.N, s.N, 1))
    return said


@functools.lru_cache(maxsize=1024)
def _linear_said(of: bytes) -> _Said:
    s = LinearShape.from_buffer_copy(of)
    said = _Said(s)
    y, bf16 = _dtype_of(s.y_dtype), _dtype_of(DTYPE_BF16)
    rows = lambda n, dtype, st: (dtype, (s.B, s.N, n), (*st, 1))  # noqa: E731
    said.x, said.dx = rows(s.in_features, bf16, s.x_stride), rows(s.in_features, bf16, s.dx_stride)
    said.y, said.z = rows(s.out_features, y, s.y_stride), rows(s.out_features, bf16, s.z_stride)
    said.residual = rows(s.out_features, y, s.residual_stride)
    said.w, said.dw = (bf16, (s.out_features, s.in_features), (s.w_stride, 1)), (bf16, (s.out_features, s.in_features), (s.dw_stride, 1))
    said.bias = (_dtype_of(s.bias_dtype), (s.out_features,), (1,))
    said.gate = (_dtype_of(s.gate_dtype), (s.B, s.out_features), (s.gate_stride, 1))
    return said


def _packed(s, stride: str, rows, features: int):
    """The record with the strides of an output that the call makes (rows on 16-byte boundaries) as ``stride``, and that output's size."""
    size = (*rows, -(-features // 8) * 8)
    steps = getattr(s, stride)
    for i in range(len(steps)):
        steps[i] = math.prod(size[i + 1:])
    return bytes(s), size


@functools.lru_cache(maxsize=1024)
def _norm_packed(of: bytes, stride: str):
    s = NormShape.from_buffer_copy(of)
    of, size = _packed(s, stride, (s.B, s.H, s.N), s.C)
    return _norm_said(of), size, s.C


@functools.lru_cache(maxsize=1024)
def _linear_packed(of: bytes):
    s = LinearShape.from_buffer_copy(of)
    of, size = _packed(s, "y_stride", (s.B, s.N), s.out_features)
    return _linear_said(of), size, s.out_features


def _room(size, features: int, dtype, device, stream):
    import torch
    t = torch.empty(size, dtype=dtype, device=device) if stream is None else _made(lambda: torch.empty(size, dtype=dtype, device=device), device, stream)
    return t if size[-1] == features else t[..., :features]


def _vector(size, device, stream):
    import torch
    return _made(lambda: torch.empty(size, dtype=torch.float32, device=device), device, stream)


def _rows_of(stride, *tensors):
    for t in tensors:
        if t is not None:
            return type(stride)(*t.stride()[:len(stride)])
    return stride


def _last_axis(t, what: str):
    if t is not None and t.shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError(f"{what}: the last axis must be contiguous")


def make_norm_shape(X, Y, weight=None, scale=None, shift=None, dX=None, eps: float = 1e-6, bias=None) -> NormShape:
    """Record of a layer norm over the last axis of X [B,H,N,C] (H = 1: whole token rows).  Y is the output of the forward
    call or the gradient dY that the backward call gets; types and strides are taken from the tensors.  shift has the
    batch stride of scale unless given; bias, which has the type of weight, is looked at only where there is no weight."""
    for t, what in ((X, "X"), (Y, "Y"), (dX, "dX")):
        if t is not None and t.dim() != 4:
            raise ValueError(f"{what} must be [B,H,N,C]")
        _last_axis(t, what)
    s = NormShape()
    s.B, s.H, s.N, s.C = X.shape
    s.x_stride, s.y_stride = _rows_of(s.x_stride, X), _rows_of(s.y_stride, Y)
    s.dy_stride, s.dx_stride = _rows_of(s.dy_stride, Y), _rows_of(s.dx_stride, dX, X)
    s.x_dtype, s.y_dtype = _dtype_code(X, "X"), _dtype_code(Y, "Y")
    affine = weight if weight is not None else bias
    s.weight_dtype = DTYPE_F32 if affine is None else _dtype_code(affine, "weight" if weight is not None else "bias")
    mod = scale if scale is not None else shift
    s.mod_dtype = DTYPE_F32 if mod is None else _dtype_code(mod, "scale")
    s.scale_stride = 0 if mod is None else mod.stride(0)
    s.shift_stride = s.scale_stride if shift is None else shift.stride(0)
    s.eps = eps
    return s


def layer_norm(X, shape: NormShape, weight=None, bias=None, shift=None, scale=None, Y=None, mean=None, rstd=None, stream=None):
    """carnator_layer_norm.  Returns Y [B,H,N,C] (its own, with rows on 16-byte boundaries, unless given); mean and rstd fp32 [B,H,N] (contiguous) are written if given."""
    dev = X.device
    if Y is None:                        # the caller's record stays as it is
        said, size, n = _norm_packed(bytes(shape), "y_stride")
        Y = _room(size, n, said.y[0], dev, stream)
    else:
        said = _norm_said(bytes(shape))
    on = _stream_on(dev, stream)
    _fit(X, "X", *said.x, dev)
    _fit(Y, "Y", *said.y, dev)
    if weight is not None:
        _fit(weight, "weight", *said.vec, dev)
    if bias is not None:
        _fit(bias, "bias", *said.vec, dev)
    if shift is not None:
        _fit(shift, "shift", *said.shift, dev)
    if scale is not None:
        _fit(scale, "scale", *said.scale, dev)
    if mean is not None:
        _fit(mean, "mean", *said.stat, dev)
    if rstd is not None:
        _fit(rstd, "rstd", *said.stat, dev)
    st = lib().carnator_layer_norm(_ptr(X), _ptr(weight), _ptr(bias), _ptr(shift), _ptr(scale), said.ref, _ptr(Y), _ptr(mean), _ptr(rstd), on)
    if st != OK:
        _check(st, "carnator_layer_norm")
    return Y


def layer_norm_backward_workspace_bytes(shape: NormShape) -> int:
    return int(lib().carnator_layer_norm_backward_workspace_bytes(ctypes.byref(shape)))


class NormGrads(NamedTuple):
    """Gradients of a layer norm; those of vectors that the norm does not have, or that were not wanted, are None."""
    dX: object
    dweight: object
    dbias: object
    dshift: object
    dscale: object


def layer_norm_backward(dY, X, mean, rstd, shape: NormShape, weight=None, bias=None, scale=None, dX=None,
                        want=("weight", "bias", "shift", "scale"), modulated=None, ws=None, stream=None) -> NormGrads:
    """carnator_layer_norm_backward.  ``want`` names the vector gradients to compute: weight (if the norm has one), bias (if
    it has a weight or a bias), shift and scale (if it has a scale, or ``modulated`` says that it has a shift only)."""
    dev = X.device
    if dX is None:
        said, size, n = _norm_packed(bytes(shape), "dx_stride")
        dX = _room(size, n, said.dx[0], dev, stream)
    else:
        said = _norm_said(bytes(shape))
    on = _stream_on(dev, stream)
    _fit(dY, "dY", *said.dy, dev)
    _fit(X, "X", *said.x, dev)
    _fit(dX, "dX", *said.dx, dev)
    _fit(mean, "mean", *said.stat, dev)
    _fit(rstd, "rstd", *said.stat, dev)
    if weight is not None:
        _fit(weight, "weight", *said.vec, dev)
    if bias is not None:
        _fit(bias, "bias", *said.vec, dev)
    if scale is not None:
        _fit(scale, "scale", *said.scale, dev)
    B, C = said.record.B, said.record.C
    dweight = dbias = dshift = dscale = None
    if weight is not None and "weight" in want:
        dweight = _vector(C, dev, stream)
    if (weight is not None or bias is not None) and "bias" in want:
        dbias = _vector(C, dev, stream)
    if scale is not None if modulated is None else modulated:
        if "shift" in want:
            dshift = _vector((B, C), dev, stream)
        if "scale" in want:
            dscale = _vector((B, C), dev, stream)
    if ws is None:
        ws = _new_ws(layer_norm_backward_workspace_bytes(said.record), dev, stream)
    elif ws.device != dev or not ws.is_contiguous():
        raise ValueError(f"ws must be contiguous and on {dev}")
    st = lib().carnator_layer_norm_backward(_ptr(dY), _ptr(X), _ptr(mean), _ptr(rstd), _ptr(weight), _ptr(bias), _ptr(scale), said.ref, _ptr(dX),
                                            _ptr(dweight), _ptr(dbias), _ptr(dshift), _ptr(dscale), _ptr(ws), ws.numel(), on)
    if st != OK:
        _check(st, "carnator_layer_norm_backward")
    return NormGrads(dX, dweight, dbias, dshift, dscale)


def make_linear_shape(X, W, Y, residual=None, Z=None, bias=None, gate=None, dX=None, dW=None, activation: int = ACT_NONE) -> LinearShape:
    """Record of Y = residual + gate * act(X W^T + bias): X [B,N,in_features], W [out_features,in_features], Y (or the dY of
    a backward call) [B,N,out_features]; types and strides are taken from the tensors."""
    for t, what, dims in ((X, "X", 3), (W, "W", 2), (Y, "Y", 3), (residual, "residual", 3), (Z, "Z", 3), (dX, "dX", 3), (dW, "dW", 2)):
        if t is not None and t.dim() != dims:
            raise ValueError(f"{what} must have {dims} axes")
        _last_axis(t, what)
    s = LinearShape()
    s.B, s.N, s.in_features = X.shape
    s.out_features = W.shape[0]
    if W.shape[1] != s.in_features or tuple(Y.shape) != (s.B, s.N, s.out_features):
        raise ValueError(f"X {tuple(X.shape)}, W {tuple(W.shape)} and Y {tuple(Y.shape)} do not belong together")
    s.x_stride, s.y_stride = _rows_of(s.x_stride, X), _rows_of(s.y_stride, Y)
    s.residual_stride, s.z_stride = _rows_of(s.residual_stride, residual, Y), _rows_of(s.z_stride, Z)
    s.dx_stride = _rows_of(s.dx_stride, dX)
    s.w_stride = W.stride(0)
    s.dw_stride = s.w_stride if dW is None else dW.stride(0)
    s.gate_stride = 0 if gate is None else gate.stride(0)
    s.activation = activation
    s.y_dtype = _dtype_code(Y, "Y")
    s.bias_dtype = DTYPE_F32 if bias is None else _dtype_code(bias, "bias")
    s.gate_dtype = DTYPE_F32 if gate is None else _dtype_code(gate, "gate")
    return s


def linear_workspace_bytes(shape: LinearShape) -> int:
    return int(lib().carnator_linear_workspace_bytes(ctypes.byref(shape)))


def linear(X, W, shape: LinearShape, bias=None, gate=None, residual=None, Y=None, Z=None, ws=None, stream=None):
    """carnator_linear.  Returns (Y [B,N,out_features] (as in layer_norm), ws); Z (bf16, the pre-activation) is written if given."""
    dev = X.device
    if Y is None:
        said, size, n = _linear_packed(bytes(shape))
        Y = _room(size, n, said.y[0], dev, stream)
    else:
        said = _linear_said(bytes(shape))
    on = _stream_on(dev, stream)
    _fit(X, "X", *said.x, dev)
    _fit(W, "W", *said.w, dev)
    _fit(Y, "Y", *said.y, dev)
    if Z is not None:
        _fit(Z, "Z", *said.z, dev)
    if residual is not None:
        _fit(residual, "residual", *said.residual, dev)
    if bias is not None:
        _fit(bias, "bias", *said.bias, dev)
    if gate is not None:
        _fit(gate, "gate", *said.gate, dev)
    if ws is None:
        ws = _new_ws(linear_workspace_bytes(said.record), dev, stream)
    elif ws.device != dev or not ws.is_contiguous():
        raise ValueError(f"ws must be contiguous and on {dev}")
    st = lib().carnator_linear(_ptr(X), _ptr(W), _ptr(bias), _ptr(gate), _ptr(residual), said.ref, _ptr(Y), _ptr(Z), _ptr(ws), ws.numel(), on)
    if st != OK:
        _check(st, "carnator_linear")
    return Y, ws


def linear_backward_workspace_bytes(shape: LinearShape) -> int:
    return int(lib().carnator_linear_backward_workspace_bytes(ctypes.byref(shape)))


class LinearGrads(NamedTuple):
    """Gradients of linear; the residual's is dY itself.  dX, dW and those not wanted are None where the call was given no room for them."""
    dX: object
    dW: object
    dbias: object
    dgate: object


def linear_backward(dY, X, W, shape: LinearShape, Z=None, gate=None, dX=None, dW=None, want=("bias", "gate"), ws=None,
                    stream=None) -> LinearGrads:
    """carnator_linear_backward.  dX (from W) and dW (from X) are computed where given (bf16); X or W that is not read may be None.
    ``want`` names the fp32 vector gradients: bias, gate (if there is one).  Z is the pre-activation that the forward call wrote."""
    dev = dY.device
    said = _linear_said(bytes(shape))
    on = _stream_on(dev, stream)
    _fit(dY, "dY", *said.y, dev)
    if (X is None and dW is not None) or (W is None and dX is not None):
        raise ValueError("dW is made from X, dX from W")
    if X is not None:
        _fit(X, "X", *said.x, dev)
    if W is not None:
        _fit(W, "W", *said.w, dev)
    if Z is not None:
        _fit(Z, "Z", *said.z, dev)
    if gate is not None:
        _fit(gate, "gate", *said.gate, dev)
    if dX is not None:
        _fit(dX, "dX", *said.dx, dev)
    if dW is not None:
        _fit(dW, "dW", *said.dw, dev)
    of = said.record
    dbias = _vector(of.out_features, dev, stream) if "bias" in want else None
    dgate = _vector((of.B, of.out_features), dev, stream) if gate is not None and "gate" in want else None
    if ws is None:
        ws = _new_ws(linear_backward_workspace_bytes(said.record), dev, stream)
    elif ws.device != dev or not ws.is_contiguous():
        raise ValueError(f"ws must be contiguous and on {dev}")
    st = lib().carnator_linear_backward(_ptr(dY), _ptr(X), _ptr(W), _ptr(Z), _ptr(gate), said.ref, _ptr(dX), _ptr(dW), _ptr(dbias), _ptr(dgate),
                                        _ptr(ws), ws.numel(), on)
    if st != OK:
        _check(st, "carnator_linear_backward")
    return LinearGrads(dX, dW, dbias, dgate)


# ---- rotary positions ---------------------------------------------------------------------------------
ROPE_INTERLEAVED, ROPE_HALF = 0, 1
ROPE_SCALE_NONE, ROPE_SCALE_LINEAR, ROPE_SCALE_BASE, ROPE_SCALE_RAMP = range(4)


def _three(v, fill):
    v = (v,) if isinstance(v, (int, float)) else tuple(v)
    if not 1 <= len(v) <= 3:
        raise ValueError("one to three axes")
    return v + (fill,) * (3 - len(v))


def rope_frequencies(pairs, theta: float = 10000.0, scaling: int = ROPE_SCALE_NONE, factor=1.0, original=0.0, low: float = 1.0, high: float = 32.0, device="cpu"):
    """carnator_rope_frequencies.  pairs, factor and original: one number, or one per axis (of factor and original, one number stands for every axis).
    Returns (float64 tensor of radians per position of every pair on ``device``, amplitude)."""
    import torch
    s = RopeScaling()
    s.pairs[:] = _three(pairs, 0)
    s.mode, s.theta, s.low, s.high = scaling, theta, low, high
    s.factor[:] = (factor,) * 3 if isinstance(factor, (int, float)) else _three(factor, 1.0)
    s.original[:] = (original,) * 3 if isinstance(original, (int, float)) else _three(original, 0.0)
    n = sum(max(p, 0) for p in s.pairs)
    freq, amplitude = (ctypes.c_double * max(n, 1))(), ctypes.c_double()
    _check(lib().carnator_rope_frequencies(ctypes.byref(s), freq, ctypes.byref(amplitude)), "carnator_rope_frequencies")
    return torch.tensor(list(freq)[:n], dtype=torch.float64, device=device), amplitude.value


def make_rope_shape(X, Y, pairs, n_text: int = 0, grid=None, positions=None, offset=(0, 0, 0), layout: int = ROPE_INTERLEAVED, amplitude: float = 1.0,
                    inverse: bool = False) -> RopeShape:
    """Record of a turn of X [B,H,N,D] into Y (None: strides of X).  pairs: pairs of channels per axis.  grid: (T, Hg, Wg) of the tokens behind n_text text tokens
    (default: one line); with positions [B or 1, N, axes] the tokens stand where it says instead.  Types and strides are taken from the tensors."""
    for t, what in ((X, "X"), (Y, "Y")):
        if t is not None and t.dim() != 4:
            raise ValueError(f"{what} must be [B,H,N,D]")
        _last_axis(t, what)
    s = RopeShape()
    s.B, s.H, s.N, s.D = X.shape
    s.x_stride, s.y_stride = _rows_of(s.x_stride, X), _rows_of(s.y_stride, Y, X)
    s.pairs[:], s.offset[:] = _three(pairs, 0), _three(offset, 0)
    s.n_text = n_text
    s.T, s.Hg, s.Wg = grid if grid is not None else (s.N - n_text, 1, 1)
    if positions is not None:
        if positions.dim() != 3 or not 1 <= positions.shape[2] <= 3 or (positions.shape[2] > 1 and positions.stride(2) != 1) or positions.shape[0] not in (1, s.B):
            raise ValueError("positions must be [B or 1, N, 1 to 3] with the last axis contiguous")
        s.axes = positions.shape[2]
        s.pos_stride[:] = [0 if positions.shape[0] == 1 else positions.stride(0), positions.stride(1)]
    s.layout, s.inverse, s.amplitude, s.x_dtype = layout, bool(inverse), amplitude, _dtype_code(X, "X")
    return s


@functools.lru_cache(maxsize=1024)
def _rope_said(of: bytes) -> _Said:
    import torch
    s = RopeShape.from_buffer_copy(of)
    said = _Said(s)
    size, x = (s.B, s.H, s.N, s.D), _dtype_of(s.x_dtype)
    said.x, said.y = (x, size, (*s.x_stride, 1)), (x, size, (*s.y_stride, 1))
    said.freq = (torch.float64, (sum(s.pairs),), (1,))
    shared = s.pos_stride[0] == 0
    said.pos = (torch.int32, (1 if shared else s.B, s.N, s.axes), (*s.pos_stride, 1))
    return said


@functools.lru_cache(maxsize=1024)
def _rope_packed(of: bytes):
    s = RopeShape.from_buffer_copy(of)
    of, size = _packed(s, "y_stride", (s.B, s.H, s.N), s.D)
    return _rope_said(of), size, s.D


def rope(X, freq, shape: RopeShape, positions=None, Y=None, stream=None):
    """carnator_rope.  freq: float64, from rope_frequencies.  Returns Y [B,H,N,D] (its own, with rows on 16-byte boundaries, unless given; may be X)."""
    dev = X.device
    if Y is None:
        said, size, n = _rope_packed(bytes(shape))
        Y = _room(size, n, said.y[0], dev, stream)
    else:
        said = _rope_said(bytes(shape))
    on = _stream_on(dev, stream)
    _fit(X, "X", *said.x, dev)
    _fit(Y, "Y", *said.y, dev)
    _fit(freq, "freq", *said.freq, dev)
    if positions is None:
        if said.record.axes:             # without them the tokens would turn as a plain line
            raise ValueError("the shape record was made with positions, the call has none")
    else:
        if said.pos[1][0] == 1 and positions.shape[0] == said.record.B and positions.stride(0) == 0:
            positions = positions[:1]              # one tensor seen by every entry
        _fit(positions, "positions", *said.pos, dev)
    st = lib().carnator_rope(_ptr(X), _ptr(freq), _ptr(positions), said.ref, _ptr(Y), on)
    if st != OK:
        _check(st, "carnator_rope")
    return Y


# ---- the end of a block and the beginning of the next one ----------------------------------------------
NORM_NONE, NORM_LAYER, NORM_RMS = 0, 1, 2


def make_block_norm_shape(R, X, S, Y, post_weight=None, post_bias=None, gate=None, weight=None, bias=None, shift=None, scale=None, dS=None, dR=None, dX=None,
                          post: int = NORM_NONE, pre: int = NORM_LAYER, post_eps: float = 1e-6, eps: float = 1e-6, residual_scale: float = 1.0) -> BlockNormShape:
    """Record of S = residual_scale R + gate post(X), Y = pre(S) modulated, all [B,N,C].  Y is the output of the forward call or the gradient dY that the backward call
    gets; dS, dR, dX are the backward call's (strides of S, S and X unless given).  Types and strides are taken from the tensors; shift has the batch stride of scale
    unless given, and the four vectors of C channels are of one type."""
    for t, what in ((R, "R"), (X, "X"), (S, "S"), (Y, "Y"), (dS, "dS"), (dR, "dR"), (dX, "dX")):
        if t is not None and t.dim() != 3:
            raise ValueError(f"{what} must be [B,N,C]")
        _last_axis(t, what)
    s = BlockNormShape()
    s.B, s.N, s.C = X.shape
    s.post, s.pre, s.post_eps, s.eps, s.residual_scale = post, pre, post_eps, eps, residual_scale
    s.r_stride, s.x_stride, s.s_stride, s.y_stride = (_rows_of(s.r_stride, t) for t in (R, X, S, Y))
    s.ds_stride, s.dr_stride, s.dx_stride = _rows_of(s.ds_stride, dS, S), _rows_of(s.dr_stride, dR, S), _rows_of(s.dx_stride, dX, X)
    stream = S if S is not None else R
    s.stream_dtype, s.x_dtype, s.y_dtype = _dtype_code(stream, "S" if S is not None else "R"), _dtype_code(X, "X"), _dtype_code(Y, "Y")
    vec = next((v for v in (post_weight, weight, post_bias, bias) if v is not None), None)
    s.weight_dtype = DTYPE_F32 if vec is None else _dtype_code(vec, "weight")
    mod = next((v for v in (gate, scale, shift) if v is not None), None)
    s.mod_dtype = DTYPE_F32 if mod is None else _dtype_code(mod, "gate, shift and scale")
    s.gate_stride = 0 if gate is None else gate.stride(0)
    rows = scale if scale is not None else shift
    s.scale_stride = 0 if rows is None else rows.stride(0)
    s.shift_stride = s.scale_stride if shift is None else shift.stride(0)
    return s


@functools.lru_cache(maxsize=1024)
def _block_said(of: bytes) -> _Said:
    s = BlockNormShape.from_buffer_copy(of)
    said = _Said(s)
    size, stream, x, y, m = (s.B, s.N, s.C), _dtype_of(s.stream_dtype), _dtype_of(s.x_dtype), _dtype_of(s.y_dtype), _dtype_of(s.mod_dtype)
    said.r, said.s, said.ds, said.dr = ((stream, size, (*st, 1)) for st in (s.r_stride, s.s_stride, s.ds_stride, s.dr_stride))
    said.x, said.dx, said.y = (x, size, (*s.x_stride, 1)), (x, size, (*s.dx_stride, 1)), (y, size, (*s.y_stride, 1))
    said.vec = (_dtype_of(s.weight_dtype), (s.C,), (1,))
    said.gate, said.shift, said.scale = ((m, (s.B, s.C), (st, 1)) for st in (s.gate_stride, s.shift_stride, s.scale_stride))
    said.stat = (_dtype_of(DTYPE_F32), (4, s.B, s.N), (s.B * s.N, s.N, 1))
    return said


@functools.lru_cache(maxsize=1024)
def _block_packed(of: bytes, strides: tuple):
    s = BlockNormShape.from_buffer_copy(of)
    for name in strides:
        of, size = _packed(s, name, (s.B, s.N), s.C)
    return _block_said(of), size, s.C


def _fit_vectors(said, dev, post_weight, post_bias, gate, weight, bias, shift, scale):
    if post_weight is not None:
        _fit(post_weight, "post_weight", *said.vec, dev)
    if post_bias is not None:
        _fit(post_bias, "post_bias", *said.vec, dev)
    if weight is not None:
        _fit(weight, "weight", *said.vec, dev)
    if bias is not None:
        _fit(bias, "bias", *said.vec, dev)
    if gate is not None:
        _fit(gate, "gate", *said.gate, dev)
    if shift is not None:
        _fit(shift, "shift", *said.shift, dev)
    if scale is not None:
        _fit(scale, "scale", *said.scale, dev)


def block_norm(R, X, shape: BlockNormShape, post_weight=None, post_bias=None, gate=None, weight=None, bias=None, shift=None, scale=None, S=None, Y=None, stats=None,
               stream=None):
    """carnator_block_norm.  Returns (S, Y) [B,N,C] (its own, with rows on 16-byte boundaries, unless given; S may be R); stats fp32 [4,B,N] is written if given."""
    dev = X.device
    if S is None or Y is None:           # the caller's record stays as it is
        said, size, n = _block_packed(bytes(shape), tuple(name for t, name in ((S, "s_stride"), (Y, "y_stride")) if t is None))
        S = _room(size, n, said.s[0], dev, stream) if S is None else S
        Y = _room(size, n, said.y[0], dev, stream) if Y is None else Y
    else:
        said = _block_said(bytes(shape))
    on = _stream_on(dev, stream)
    _fit(R, "R", *said.r, dev)
    _fit(X, "X", *said.x, dev)
    _fit(S, "S", *said.s, dev)
    _fit(Y, "Y", *said.y, dev)
    _fit_vectors(said, dev, post_weight, post_bias, gate, weight, bias, shift, scale)
    if stats is not None:
        _fit(stats, "stats", *said.stat, dev)
    st = lib().carnator_block_norm(_ptr(R), _ptr(X), _ptr(post_weight), _ptr(post_bias), _ptr(gate), _ptr(weight), _ptr(bias), _ptr(shift), _ptr(scale), said.ref,
                                   _ptr(S), _ptr(Y), _ptr(stats), on)
    if st != OK:
        _check(st, "carnator_block_norm")
    return S, Y


def block_norm_backward_workspace_bytes(shape: BlockNormShape) -> int:
    return int(lib().carnator_block_norm_backward_workspace_bytes(ctypes.byref(shape)))


class BlockNormGrads(NamedTuple):
    """Gradients of block_norm; those of vectors that it does not have, or that were not wanted, are None."""
    dR: object
    dX: object
    dpost_weight: object
    dpost_bias: object
    dgate: object
    dweight: object
    dbias: object
    dshift: object
    dscale: object


def block_norm_backward(dY, S, X, stats, shape: BlockNormShape, dS=None, post_weight=None, post_bias=None, gate=None, weight=None, bias=None, scale=None, dR=None, dX=None,
                        want=("post_weight", "post_bias", "gate", "weight", "bias", "shift", "scale"), modulated=None, ws=None, stream=None) -> BlockNormGrads:
    """carnator_block_norm_backward.  ``want`` names the vector gradients to compute, of those that there are: post_weight, post_bias, gate, weight, bias, and shift and
    scale (if there is a scale, or ``modulated`` says that there is a shift only)."""
    dev = X.device
    if dR is None or dX is None:
        said, size, n = _block_packed(bytes(shape), tuple(name for t, name in ((dR, "dr_stride"), (dX, "dx_stride")) if t is None))
        dR = _room(size, n, said.dr[0], dev, stream) if dR is None else dR
        dX = _room(size, n, said.dx[0], dev, stream) if dX is None else dX
    else:
        said = _block_said(bytes(shape))
    on = _stream_on(dev, stream)
    _fit(dY, "dY", *said.y, dev)
    _fit(S, "S", *said.s, dev)
    _fit(X, "X", *said.x, dev)
    _fit(dR, "dR", *said.dr, dev)
    _fit(dX, "dX", *said.dx, dev)
    _fit(stats, "stats", *said.stat, dev)
    if dS is not None:
        _fit(dS, "dS", *said.ds, dev)
    _fit_vectors(said, dev, post_weight, post_bias, gate, weight, bias, None, scale)
    B, C = said.record.B, said.record.C

    mod = scale is not None if modulated is None else modulated
    # fp32, where the tensors are: the quickest way to a tensor, and a small call's time is the host's
    new = stats.new_empty if stream is None else lambda *size: _vector(size, dev, stream)
    dpw = new(C) if post_weight is not None and "post_weight" in want else None
    dpb = new(C) if post_bias is not None and "post_bias" in want else None
    dg = new(B, C) if gate is not None and "gate" in want else None
    dw = new(C) if weight is not None and "weight" in want else None
    db = new(C) if bias is not None and "bias" in want else None
    dsh = new(B, C) if mod and "shift" in want else None
    dsc = new(B, C) if mod and "scale" in want else None
    if ws is None:
        ws = _new_ws(block_norm_backward_workspace_bytes(said.record), dev, stream)
    elif ws.device != dev or not ws.is_contiguous():
        raise ValueError(f"ws must be contiguous and on {dev}")
    st = lib().carnator_block_norm_backward(_ptr(dY), _ptr(dS), _ptr(S), _ptr(X), _ptr(stats), _ptr(post_weight), _ptr(post_bias), _ptr(gate), _ptr(weight), _ptr(bias),
                                            _ptr(scale), said.ref, _ptr(dR), _ptr(dX), _ptr(dpw), _ptr(dpb), _ptr(dg), _ptr(dw), _ptr(db), _ptr(dsh), _ptr(dsc),
                                            _ptr(ws), ws.numel(), on)
    if st != OK:
        _check(st, "carnator_block_norm_backward")
    return BlockNormGrads(dR, dX, dpw, dpb, dg, dw, db, dsh, dsc)


# ---- 8-bit operands and their product ---------------------------------------------------------------------
FP8_BLOCK = 128                # in_features (and out_features of a weight) that share a scale


def _x_code(t, what: str) -> int:
    import torch
    return DTYPE_E4M3 if t.dtype == torch.float8_e4m3fn else _dtype_code(t, what)


def make_quantize_shape(X, Q, scale, block_rows: int = 1) -> QuantizeShape:
    """Record of X [B,N,K] taken to e4m3 Q [B,N,K] with scale fp32 [B, N or ceil(N/128), ceil(K/128)]; block_rows 1 (activations) or 128 (a weight).
    Q and scale may be None: rows on 16-byte boundaries; scales of neighbouring rows (activations) or columns (a weight) beside each other."""
    for t, what in ((X, "X"), (Q, "Q"), (scale, "scale")):
        if t is not None and t.dim() != 3:
            raise ValueError(f"{what} must have 3 axes")
    _last_axis(X, "X")
    _last_axis(Q, "Q")
    s = QuantizeShape()
    s.B, s.N, s.K = X.shape
    s.block_rows, s.x_dtype = block_rows, _dtype_code(X, "X")
    wide, blocks, rows = -(-s.K // 16) * 16, -(-s.K // FP8_BLOCK), -(-s.N // max(block_rows, 1))
    s.x_stride = _rows_of(s.x_stride, X)
    s.q_stride[:] = (s.N * wide, wide) if Q is None else Q.stride()[:2]
    s.scale_stride[:] = scale.stride() if scale is not None else (rows * blocks, 1, rows) if block_rows == 1 else (rows * blocks, blocks, 1)
    return s


@functools.lru_cache(maxsize=1024)
def _quantize_said(of: bytes) -> _Said:
    import torch
    s = QuantizeShape.from_buffer_copy(of)
    said = _Said(s)
    size = (s.B, s.N, s.K)
    said.x, said.q = (_dtype_of(s.x_dtype), size, (*s.x_stride, 1)), (torch.float8_e4m3fn, size, (*s.q_stride, 1))
    said.scale = (torch.float32, (s.B, -(-s.N // max(s.block_rows, 1)), -(-s.K // FP8_BLOCK)), tuple(s.scale_stride))
    return said


def _room_as(dtype, size, stride, device, stream):
    import torch
    return _made(lambda: torch.empty_strided(size, stride, dtype=dtype, device=device), device, stream)


def quantize_fp8(X, shape: QuantizeShape, Q=None, scale=None, stream=None):
    """carnator_quantize_fp8.  Returns (Q float8_e4m3fn [B,N,K], scale fp32); those not given are made with the record's strides."""
    dev = X.device
    said = _quantize_said(bytes(shape))
    on = _stream_on(dev, stream)
    _fit(X, "X", *said.x, dev)
    if Q is None:
        Q = _room_as(*said.q, dev, stream)
    else:
        _fit(Q, "Q", *said.q, dev)
    if scale is None:
        scale = _room_as(*said.scale, dev, stream)
    else:
        _fit(scale, "scale", *said.scale, dev)
    st = lib().carnator_quantize_fp8(_ptr(X), said.ref, _ptr(Q), _ptr(scale), on)
    if st != OK:
        _check(st, "carnator_quantize_fp8")
    return Q, scale


def make_linear_fp8_shape(X, W, w_scale, Y, x_scale=None, residual=None, bias=None, gate=None, activation: int = ACT_NONE) -> LinearFp8Shape:
    """Record of Y = residual + gate * act(X W^T + bias) with W e4m3 [out_features,in_features] and w_scale fp32 [ceil(out/128), ceil(in/128)]; X [B,N,in_features]
    is e4m3 with x_scale fp32 [B,N,ceil(in/128)], or float32 / bfloat16 without.  Types and strides are taken from the tensors."""
    import torch
    for t, what, dims in ((X, "X", 3), (W, "W", 2), (Y, "Y", 3), (residual, "residual", 3), (x_scale, "x_scale", 3), (w_scale, "w_scale", 2)):
        if t is not None and t.dim() != dims:
            raise ValueError(f"{what} must have {dims} axes")
        if t is not x_scale and t is not w_scale:
            _last_axis(t, what)
    s = LinearFp8Shape()
    s.B, s.N, s.in_features = X.shape
    s.out_features = W.shape[0]
    if W.shape[1] != s.in_features or tuple(Y.shape) != (s.B, s.N, s.out_features):
        raise ValueError(f"X {tuple(X.shape)}, W {tuple(W.shape)} and Y {tuple(Y.shape)} do not belong together")
    if W.dtype != torch.float8_e4m3fn:
        raise ValueError(f"W must be float8_e4m3fn, not {W.dtype}")
    s.x_dtype = _x_code(X, "X")
    if (x_scale is not None) != (s.x_dtype == DTYPE_E4M3):
        raise ValueError("an 8-bit X comes with x_scale, any other without")
    s.x_stride, s.y_stride = _rows_of(s.x_stride, X), _rows_of(s.y_stride, Y)
    s.residual_stride = _rows_of(s.residual_stride, residual, Y)
    s.w_stride = W.stride(0)
    if x_scale is not None:
        s.x_scale_stride[:] = x_scale.stride()
    s.w_scale_stride[:] = w_scale.stride()
    s.gate_stride = 0 if gate is None else gate.stride(0)
    s.activation = activation
    s.y_dtype = _dtype_code(Y, "Y")
    s.bias_dtype = DTYPE_F32 if bias is None else _dtype_code(bias, "bias")
    s.gate_dtype = DTYPE_F32 if gate is None else _dtype_code(gate, "gate")
    return s


@functools.lru_cache(maxsize=1024)
def _linear_fp8_said(of: bytes) -> _Said:
    import torch
    s = LinearFp8Shape.from_buffer_copy(of)
    said = _Said(s)
    y, blocks = _dtype_of(s.y_dtype), -(-s.in_features // FP8_BLOCK)
    said.x = (_dtype_of(s.x_dtype), (s.B, s.N, s.in_features), (*s.x_stride, 1))
    said.y, said.residual = ((y, (s.B, s.N, s.out_features), (*st, 1)) for st in (s.y_stride, s.residual_stride))
    said.w = (torch.float8_e4m3fn, (s.out_features, s.in_features), (s.w_stride, 1))
    said.x_scale = (torch.float32, (s.B, s.N, blocks), tuple(s.x_scale_stride))
    said.w_scale = (torch.float32, (-(-s.out_features // FP8_BLOCK), blocks), tuple(s.w_scale_stride))
    said.bias = (_dtype_of(s.bias_dtype), (s.out_features,), (1,))
    said.gate = (_dtype_of(s.gate_dtype), (s.B, s.out_features), (s.gate_stride, 1))
    return said


@functools.lru_cache(maxsize=1024)
def _linear_fp8_packed(of: bytes):
    s = LinearFp8Shape.from_buffer_copy(of)
    of, size = _packed(s, "y_stride", (s.B, s.N), s.out_features)
    return _linear_fp8_said(of), size, s.out_features


def linear_fp8_workspace_bytes(shape: LinearFp8Shape) -> int:
    return int(lib().carnator_linear_fp8_workspace_bytes(ctypes.byref(shape)))


def linear_fp8(X, W, w_scale, shape: LinearFp8Shape, x_scale=None, bias=None, gate=None, residual=None, Y=None, ws=None, stream=None):
    """carnator_linear_fp8.  Returns (Y [B,N,out_features] (as in layer_norm), ws)."""
    dev = X.device
    if Y is None:
        said, size, n = _linear_fp8_packed(bytes(shape))
        Y = _room(size, n, said.y[0], dev, stream)
    else:
        said = _linear_fp8_said(bytes(shape))
    on = _stream_on(dev, stream)
    _fit(X, "X", *said.x, dev)
    _fit(W, "W", *said.w, dev)
    _fit(w_scale, "w_scale", *said.w_scale, dev)
    _fit(Y, "Y", *said.y, dev)
    if x_scale is not None:
        _fit(x_scale, "x_scale", *said.x_scale, dev)
    if residual is not None:
        _fit(residual, "residual", *said.residual, dev)
    if bias is not None:
        _fit(bias, "bias", *said.bias, dev)
    if gate is not None:
        _fit(gate, "gate", *said.gate, dev)
    if ws is None:
        ws = _new_ws(linear_fp8_workspace_bytes(said.record), dev, stream)
    elif ws.device != dev or not ws.is_contiguous():
        raise ValueError(f"ws must be contiguous and on {dev}")
    st = lib().carnator_linear_fp8(_ptr(X), _ptr(x_scale), _ptr(W), _ptr(w_scale), _ptr(bias), _ptr(gate), _ptr(residual), said.ref, _ptr(Y), _ptr(ws), ws.numel(), on)
    if st != OK:
        _check(st, "carnator_linear_fp8")
    return Y, ws


# ---- host-side scalars (no GPU) ---------------------------------------------------------------------
def delta_e00(lab_a, lab_b) -> float:
    a = (ctypes.c_double * 3)(*[float(x) for x in lab_a])
    b = (ctypes.c_double * 3)(*[float(x) for x in lab_b])
    return float(lib().carnator_delta_e00(a, b))


def context_discrepancy(labs_q, labs_j) -> float:
    """labs_q, labs_j: equally long sequences of (L*, a*, b*) triples, one per shared noun."""
    n = len(labs_q)
    if n != len(labs_j):
        raise ValueError("one colour per shared noun on both sides")
    a = (ctypes.c_double * (3 * n))(*[float(x) for c in labs_q for x in c])
    b = (ctypes.c_double * (3 * n))(*[float(x) for c in labs_j for x in c])
    return float(lib().carnator_context_discrepancy(a, b, n))


def size_discrepancy(area_q: float, area_j: float) -> float:
    return float(lib().carnator_size_discrepancy(float(area_q), float(area_j)))


def shape_discrepancy(m_q, m_j, resolution: int = 32) -> float:
    """m_q, m_j: 2-D numpy uint8 indicators."""
    import numpy as np
    a = np.ascontiguousarray(m_q, dtype=np.uint8)
    b = np.ascontiguousarray(m_j, dtype=np.uint8)
    return float(lib().carnator_shape_discrepancy(a.ctypes.data, a.shape[0], a.shape[1], b.ctypes.data, b.shape[0], b.shape[1],
                                                  int(resolution)))


def compatibility_gate(d, tau, applicable=None) -> int:
    n = len(d)
    dd = (ctypes.c_double * n)(*[float(x) for x in d])
    tt = (ctypes.c_double * n)(*[float(x) for x in tau])
    ap = None
    if applicable is not None:
        ap = (ctypes.c_uint8 * n)(*[int(bool(x)) for x in applicable])
    return int(lib().carnator_compatibility_gate(dd, tt, ap, n))


def clopper_pearson_upper(unsafe: int, accepted: int, alpha: float) -> float:
    return float(lib().carnator_clopper_pearson_upper(int(unsafe), int(accepted), float(alpha)))
