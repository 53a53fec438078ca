"""ctypes binding of libqrm.so: same names as the C ABI (include/qrm.h), argument marshalling only.

Tensors are torch CUDA(ROCm) tensors used purely as device memory; streams are torch streams.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional

import numpy as np

QRM_OK, QRM_E_INVALID, QRM_E_UNSUPPORTED, QRM_E_NOMEM, QRM_E_DEVICE = 0, 1, 2, 3, 4

_HERE = os.path.dirname(os.path.abspath(__file__))
# QRM_LIBRARY selects another build of the same library (same ABI), e.g. one with different tuning constants
_LIB_PATH = os.environ.get("QRM_LIBRARY") or os.path.join(_HERE, "libqrm.so")
_lib = None


class QrmError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"qrm status {status}: {message}")
        self.status = status
        self.message = message


class _ExtDesc(C.Structure):
    _fields_ = [("in_ch", C.c_int32), ("n_blocks", C.c_int32), ("channels", C.c_int32), ("n_bits", C.c_int32),
                ("conv_w", C.POINTER(C.c_float)), ("scale", C.POINTER(C.c_float)), ("bias", C.POINTER(C.c_float)),
                ("final_affine", C.c_int32), ("final_relu", C.c_int32),
                ("lin_w", C.POINTER(C.c_float)), ("lin_b", C.POINTER(C.c_float)),
                ("mean", C.c_float * 3), ("std", C.c_float * 3)]


class _RsDesc(C.Structure):
    _fields_ = [("m", C.c_int32), ("prim_poly", C.c_uint32), ("n", C.c_int32), ("k", C.c_int32), ("fcr", C.c_int32)]


class _GroupNormDesc(C.Structure):
    _fields_ = [("N", C.c_int64), ("P", C.c_int64), ("C", C.c_int32), ("groups", C.c_int32), ("type", C.c_int32), ("act", C.c_int32),
                ("eps", C.c_float), ("x_pixel", C.c_int64), ("x_image", C.c_int64), ("y_pixel", C.c_int64), ("y_image", C.c_int64)]
    _maps = None

    def __setattr__(self, name, value):
        super().__setattr__(name, value)
        if name != "_maps":
            super().__setattr__("_maps", None)

    def maps(self):
        """What the call's tensors have to be: (dtype or None, shape of a map, strides of x, strides of y, statistics), read once."""
        if self._maps is None:
            N, P, C_ = self.N, self.P, self.C
            strides = [(image or P * (pixel or C_), pixel or C_, 1) for pixel, image in ((self.x_pixel, self.x_image), (self.y_pixel, self.y_image))]
            self._maps = (_kinds().dtypes.get(self.type), (N, P, C_), *strides, N * self.groups)
        return self._maps


class _AttentionDesc(C.Structure):
    _fields_ = [("N", C.c_int64), ("Lq", C.c_int64), ("Lk", C.c_int64), ("heads", C.c_int32), ("kv_heads", C.c_int32), ("D", C.c_int32),
                ("type", C.c_int32), ("causal", C.c_int32), ("scale", C.c_float)] + \
               [(f"{t}_{s}", C.c_int64) for t in "qkvo" for s in ("row", "head", "image")]
    _rows = None

    def __setattr__(self, name, value):
        super().__setattr__(name, value)
        if name != "_rows":
            super().__setattr__("_rows", None)

    def rows(self):
        """What the call's tensors have to be: (dtype or None, {tensor: (shape, strides)} of q, k, v, o, numbers of lse), read once."""
        if self._rows is None:
            lie = {}
            for t in "qkvo":
                shape = (self.N, self.Lk, self.kv_heads, self.D) if t in "kv" else (self.N, self.Lq, self.heads, self.D)
                row = getattr(self, t + "_row") or shape[2] * shape[3]
                lie[t] = (shape, (getattr(self, t + "_image") or max(shape[1], 1) * row, row, getattr(self, t + "_head") or shape[3], 1))
            self._rows = (_kinds().dtypes.get(self.type), lie, self.N * self.heads * self.Lq)
        return self._rows


class _AdamwTensor(C.Structure):
    _fields_ = [("n", C.c_int64), ("d_param", C.c_void_p), ("d_m", C.c_void_p), ("d_v", C.c_void_p), ("d_m_scale", C.c_void_p),
                ("d_v_scale", C.c_void_p), ("d_copy", C.c_void_p), ("weight_decay", C.c_float), ("lr_scale", C.c_float)]


class _AdamwDesc(C.Structure):
    _fields_ = [("n_tensors", C.c_int32), ("param_type", C.c_int32), ("grad_type", C.c_int32), ("copy_type", C.c_int32),
                ("state_bits", C.c_int32)]


EXPORTS = ["qrm_create", "qrm_destroy", "qrm_last_error", "qrm_set_micro_batch", "qrm_workspace_bytes",
           "qrm_extract_tiles", "qrm_preprocess", "qrm_select_tiles_variance", "qrm_extractor_forward", "qrm_extractor_blocks", "qrm_rs_decode", "qrm_detect",
           "qrm_detect_host", "qrm_plan_streams", "qrm_key_threshold", "qrm_set_key", "qrm_verify_key", "qrm_detect_verify",
           "qrm_profile_enable", "qrm_profile_read", "qrm_profile_read_chunks", "qrm_release_stream", "qrm_detect_static", "qrm_version",
           "qrm_group_norm", "qrm_group_norm_backward", "qrm_adamw_create", "qrm_adamw_destroy", "qrm_adamw_step", "qrm_unpack_moment",
           "qrm_message_loss", "qrm_attention", "qrm_attention_backward", "qrm_adamw_grad_norm", "qrm_adamw_scale_grads"]
DIAG_EXPORTS = ["qrm_diag_set_flags", "qrm_diag_matrix_rate", "qrm_diag_pair_split",
                "qrm_diag_wide_schedule", "qrm_diag_last_lines", "qrm_diag_host_plan",
                "qrm_diag_preprocess_strips", "qrm_diag_rs_lanes", "qrm_diag_chain_patience", "qrm_diag_chain_count",
                "qrm_diag_chain_left_over", "qrm_diag_chain_rule", "qrm_diag_workspace"]   # include/qrm_diag.h: bench and test tooling

QRM_MAX_STREAMS = 8   # include/qrm.h
QRM_F32, QRM_BF16, QRM_F16 = 0, 1, 2
QRM_ACT_NONE, QRM_ACT_RELU, QRM_ACT_SILU = 0, 1, 2
QRM_MOMENT_BLOCK = 256
QRM_ATTENTION_MAX_D = 512
ACTIVATIONS = {"none": QRM_ACT_NONE, "relu": QRM_ACT_RELU, "silu": QRM_ACT_SILU}
QRM_DIAG_NO_FUSED_PAIRS, QRM_DIAG_POISON_WORKSPACE, QRM_DIAG_FUSE_ALWAYS, QRM_DIAG_CHAIN_ALWAYS, QRM_DIAG_NO_CHAIN = 1, 2, 4, 8, 16
(QRM_PROFILE_PAIR_FIRST, QRM_PROFILE_PAIR_MID, QRM_PROFILE_PAIR_LAST, QRM_PROFILE_BLOCK_FIRST, QRM_PROFILE_BLOCK_MID,
 QRM_PROFILE_BLOCK_LAST, QRM_PROFILE_HEAD, QRM_PROFILE_RS_DECODE, QRM_PROFILE_CHAIN, QRM_PROFILE_KINDS) = range(10)
PROFILE_KIND_NAMES = ["pair_first", "pair_mid", "pair_last", "block_first", "block_mid", "block_last", "head", "rs_decode", "chain"]


def lib_path() -> str:
    return _LIB_PATH


def load_library():
    """Load libqrm.so; building is the job of build.py / __graft_entry__.build(), not of the import."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise ImportError(f"{_LIB_PATH} is missing: run `python -m paper_2509_02447_amd.build` "
                          "(there is no CPU fallback)")
    lib = C.CDLL(_LIB_PATH)
    vp, i32, i64 = C.c_void_p, C.c_int32, C.c_int64
    lib.qrm_create.argtypes = [C.POINTER(_ExtDesc), C.POINTER(_RsDesc), C.c_int, C.POINTER(vp)]
    lib.qrm_create.restype = C.c_int
    lib.qrm_destroy.argtypes = [vp]
    lib.qrm_destroy.restype = None
    lib.qrm_last_error.argtypes = [vp]
    lib.qrm_last_error.restype = C.c_char_p
    lib.qrm_set_micro_batch.argtypes = [vp, i32]
    lib.qrm_set_micro_batch.restype = C.c_int
    lib.qrm_workspace_bytes.argtypes = [vp, i64, i32, i32]
    lib.qrm_workspace_bytes.restype = C.c_size_t
    lib.qrm_extract_tiles.argtypes = [vp, vp, i64, i32, i32, vp, i32, vp, vp]
    lib.qrm_extract_tiles.restype = C.c_int
    lib.qrm_preprocess.argtypes = [vp, vp, i64, i32, i32, i32, vp, i32, vp, vp]
    lib.qrm_preprocess.restype = C.c_int
    lib.qrm_select_tiles_variance.argtypes = [vp, vp, i64, i32, i32, i32, i32, vp, vp, vp]
    lib.qrm_select_tiles_variance.restype = C.c_int
    lib.qrm_extractor_forward.argtypes = [vp, vp, i64, i32, i32, vp, vp, vp]
    lib.qrm_extractor_forward.restype = C.c_int
    lib.qrm_extractor_blocks.argtypes = [vp, vp, i64, i32, i32, i32, vp, vp]
    lib.qrm_extractor_blocks.restype = C.c_int
    lib.qrm_rs_decode.argtypes = [vp, vp, i64, vp, vp, vp, vp]
    lib.qrm_rs_decode.restype = C.c_int
    lib.qrm_detect.argtypes = [vp, vp, i64, i32, i32, vp, i32, vp, vp, vp, vp, vp, vp]
    lib.qrm_detect.restype = C.c_int
    lib.qrm_detect_static.argtypes = [vp, vp, i64, i32, i32, vp, i32, vp, vp, vp, vp, vp, vp]
    lib.qrm_detect_static.restype = C.c_int
    lib.qrm_detect_host.argtypes = [vp, C.POINTER(vp), i32, i32, i32, i32, C.POINTER(vp), i32, i32, vp, vp, vp]
    lib.qrm_detect_host.restype = C.c_int
    lib.qrm_key_threshold.argtypes = [i32, C.c_double]
    lib.qrm_key_threshold.restype = C.c_int32
    lib.qrm_plan_streams.argtypes = [i32, C.POINTER(C.c_double), C.POINTER(C.c_double), i64, i64, i32, C.c_double,
                                     C.c_double, i32, C.POINTER(i32), C.POINTER(i64), C.POINTER(C.c_double),
                                     C.POINTER(i32)]
    lib.qrm_plan_streams.restype = C.c_int
    lib.qrm_set_key.argtypes = [vp, vp, i32]
    lib.qrm_set_key.restype = C.c_int
    lib.qrm_verify_key.argtypes = [vp, vp, i64, vp, vp, vp]
    lib.qrm_verify_key.restype = C.c_int
    lib.qrm_detect_verify.argtypes = [vp, vp, i64, i32, i32, vp, i32, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.qrm_detect_verify.restype = C.c_int
    lib.qrm_profile_enable.argtypes = [vp, i32]
    lib.qrm_profile_enable.restype = C.c_int
    lib.qrm_profile_read.argtypes = [vp, i32, C.POINTER(C.c_double), C.POINTER(C.c_int64), C.POINTER(C.c_double)]
    lib.qrm_profile_read.restype = C.c_int
    lib.qrm_profile_read_chunks.argtypes = [vp, i32, C.POINTER(C.c_double), C.POINTER(i32)]
    lib.qrm_profile_read_chunks.restype = C.c_int
    lib.qrm_release_stream.argtypes = [vp, vp]
    lib.qrm_release_stream.restype = C.c_int
    lib.qrm_diag_set_flags.argtypes = [vp, i32]
    lib.qrm_diag_set_flags.restype = C.c_int
    lib.qrm_diag_matrix_rate.argtypes = [vp, i32, C.POINTER(C.c_double)]
    lib.qrm_diag_matrix_rate.restype = C.c_int
    lib.qrm_diag_pair_split.argtypes = [i32] * 5 + [C.POINTER(i32)] * 3
    lib.qrm_diag_pair_split.restype = C.c_int
    lib.qrm_diag_wide_schedule.argtypes = [i32] * 4 + [C.POINTER(i32), C.POINTER(C.c_double), C.POINTER(C.c_double)]
    lib.qrm_diag_wide_schedule.restype = C.c_int
    lib.qrm_diag_last_lines.argtypes = [i32] * 5 + [C.POINTER(i32), C.POINTER(i64)]
    lib.qrm_diag_last_lines.restype = C.c_int
    lib.qrm_diag_host_plan.argtypes = [i32] * 8 + [C.POINTER(i32)] * 3
    lib.qrm_diag_host_plan.restype = C.c_int
    lib.qrm_diag_preprocess_strips.argtypes = [i64, i32, C.POINTER(i32)]
    lib.qrm_diag_preprocess_strips.restype = C.c_int
    lib.qrm_diag_rs_lanes.argtypes = [i32, i32, i64, C.POINTER(i32)]
    lib.qrm_diag_rs_lanes.restype = C.c_int
    lib.qrm_diag_chain_patience.argtypes = [vp, i32]
    lib.qrm_diag_chain_patience.restype = C.c_int
    lib.qrm_diag_chain_count.argtypes = [vp, vp, i32, i32, C.c_uint32]
    lib.qrm_diag_chain_count.restype = C.c_int
    lib.qrm_diag_chain_left_over.argtypes = [vp, vp, i32, C.c_uint32]
    lib.qrm_diag_chain_left_over.restype = C.c_int
    lib.qrm_diag_chain_rule.argtypes = [i32] * 6 + [C.POINTER(i32)] * 2
    lib.qrm_diag_chain_rule.restype = C.c_int
    lib.qrm_diag_workspace.argtypes = [vp, vp, C.POINTER(vp), C.POINTER(i64), C.POINTER(i32)]
    lib.qrm_diag_workspace.restype = C.c_int
    lib.qrm_group_norm.argtypes = [vp, C.POINTER(_GroupNormDesc)] + [vp] * 7
    lib.qrm_group_norm.restype = C.c_int
    lib.qrm_group_norm_backward.argtypes = [vp, C.POINTER(_GroupNormDesc)] + [vp] * 10
    lib.qrm_group_norm_backward.restype = C.c_int
    lib.qrm_adamw_create.argtypes = [vp, C.POINTER(_AdamwDesc), C.POINTER(_AdamwTensor), C.POINTER(vp)]
    lib.qrm_adamw_create.restype = C.c_int
    lib.qrm_adamw_destroy.argtypes = [vp]
    lib.qrm_adamw_destroy.restype = None
    lib.qrm_adamw_step.argtypes = [vp, vp, C.POINTER(vp), i64, C.c_double, C.c_double, C.c_double, C.c_double, vp, vp]
    lib.qrm_adamw_step.restype = C.c_int
    lib.qrm_unpack_moment.argtypes = [vp, i32, vp, vp, i64, i32, vp, vp]
    lib.qrm_unpack_moment.restype = C.c_int
    lib.qrm_message_loss.argtypes = [vp, vp, vp, i64, i64, i32, C.c_float, vp, vp, vp, vp, vp]
    lib.qrm_message_loss.restype = C.c_int
    lib.qrm_attention.argtypes = [vp, C.POINTER(_AttentionDesc)] + [vp] * 8
    lib.qrm_attention.restype = C.c_int
    lib.qrm_attention_backward.argtypes = [vp, C.POINTER(_AttentionDesc)] + [vp] * 12
    lib.qrm_attention_backward.restype = C.c_int
    lib.qrm_adamw_grad_norm.argtypes = [vp, vp, C.POINTER(vp), C.c_double, vp, vp, vp, vp]
    lib.qrm_adamw_grad_norm.restype = C.c_int
    lib.qrm_adamw_scale_grads.argtypes = [vp, vp, C.POINTER(vp), vp, C.POINTER(vp), vp]
    lib.qrm_adamw_scale_grads.restype = C.c_int
    lib.qrm_version.argtypes = []
    lib.qrm_version.restype = C.c_char_p
    _lib = lib
    return lib


def version() -> str:
    return load_library().qrm_version().decode()


def qrm_key_threshold(n_bits: int, fpr: float) -> int:
    return int(load_library().qrm_key_threshold(int(n_bits), float(fpr)))


def qrm_plan_streams(t, u, B: int, b0: int, P: int, M_cap: float, eps: float, tau: int):
    """-> (status, s list, m list, J, accepted): streams and micro-batch per stage (host-only)."""
    K = len(t)
    ta, ua = (C.c_double * K)(*[float(x) for x in t]), (C.c_double * K)(*[float(x) for x in u])
    s, m = (C.c_int32 * K)(), (C.c_int64 * K)()
    J, acc = C.c_double(0.0), C.c_int32(0)
    st = load_library().qrm_plan_streams(K, ta, ua, int(B), int(b0), int(P), float(M_cap), float(eps), int(tau), s, m,
                                         C.byref(J), C.byref(acc))
    return int(st), list(s), list(m), float(J.value), int(acc.value)


def _fptr(a: Optional[np.ndarray]):
    if a is None:
        return None
    return a.ctypes.data_as(C.POINTER(C.c_float))


def _dptr(t) -> Optional[int]:
    """Device pointer of a torch tensor (or None)."""
    if t is None:
        return None
    assert t.is_cuda and t.is_contiguous(), "device tensors must be contiguous and on the GPU"
    return t.data_ptr()


class _Kinds:
    """The torch dtypes that calls take, known once a caller has torch."""
    _known = None

    def __init__(self):
        import torch
        self.f32, self.i32 = torch.float32, torch.int32
        self.codes = {torch.float32: QRM_F32, torch.bfloat16: QRM_BF16, torch.float16: QRM_F16}
        self.dtypes = {code: dtype for dtype, code in self.codes.items()}


def _kinds() -> _Kinds:
    if _Kinds._known is None:
        _Kinds._known = _Kinds()
    return _Kinds._known


def _dptr_of(t, dtype, n: int) -> Optional[int]:
    """Device pointer of a contiguous tensor of at least n elements of a dtype (or None)."""
    if t is None:
        return None
    assert t.dtype is dtype and t.numel() >= n and t.is_cuda and t.is_contiguous(), \
        "device tensors must be of the type and of at least the size that the call takes, contiguous and on the GPU"
    return t.data_ptr()


def _dptr_bytes(t, n: int) -> Optional[int]:
    """The same of elements of one byte, whatever they are called."""
    if t is None:
        return None
    assert t.element_size() == 1 and t.numel() >= n and t.is_cuda and t.is_contiguous(), \
        "device tensors must have one byte an element and at least the size that the call takes, be contiguous and on the GPU"
    return t.data_ptr()


def _lies(t, N: int, P: int, C: int, pixel: int, image: int) -> bool:
    """Whether channel c of pixel p of image i of a map [..,C] lies i * image + p * pixel + c elements from its first one.  The tensor's
    channels may be more than C and its images more than N; pixels may have several dimensions."""
    if N < 1 or P < 1 or C < 1:                              # no images, or refused
        return True
    if pixel == C and (image == P * C or N == 1) and t.numel() == N * P * C and t.is_contiguous():
        return True
    shape, stride = t.shape, t.stride()
    if len(shape) < 2:                                       # a buffer
        return t.is_contiguous() and t.numel() >= (N - 1) * image + (P - 1) * pixel + C
    if shape[-1] < C or (C > 1 and stride[-1] != 1):
        return False
    inside, left = 1, N * P                                  # pixels of the dimensions so far
    for k in range(len(shape) - 2, -1, -1):
        size = min(shape[k], left // inside) if k == 0 else shape[k]
        if size > 1:
            whole = inside % P == 0                          # of images; else of pixels, which end with the image unless images follow as pixels do
            if stride[k] != (image * (inside // P) if whole else pixel * inside) or not (whole or P % (inside * size) == 0 or image == P * pixel or N <= 1):
                return False
        inside *= size
    return inside == left


def _dptr_map(t, dtype, shape, strides) -> Optional[int]:
    """Device pointer of a map [N,P,C] that lies as its descriptor says (or None)."""
    if t is None:
        return None
    if t.dtype is dtype and t.is_cuda and t.stride() == strides and t.shape == shape:
        return t.data_ptr()
    assert t.is_cuda, "device tensors must be on the GPU"
    # (a dtype of None: a descriptor that is refused)
    assert (t.dtype is dtype or dtype is None) and _lies(t, *shape, strides[1], strides[0]), "a map has another type, size or strides than its descriptor"
    return t.data_ptr()


def type_code(dtype) -> int:
    """qrm_type of a torch dtype."""
    return _kinds().codes[dtype]


def group_norm_desc(N: int, P: int, C: int, groups: int, dtype, act: str = "none", eps: float = 1e-6, x_pixel: int = 0,
                    x_image: int = 0, y_pixel: int = 0, y_image: int = 0):
    """The qrm_group_norm_desc of maps [N,P,C] of `dtype`; act is "none", "relu" or "silu"; strides in elements, 0 = dense."""
    return _GroupNormDesc(int(N), int(P), int(C), int(groups), type_code(dtype), ACTIVATIONS[act], float(eps), int(x_pixel),
                          int(x_image), int(y_pixel), int(y_image))


def _dptr_rows(t, dtype, lie) -> Optional[int]:
    """Device pointer of rows [N,L,heads,D] that lie as their descriptor says (or None); a buffer of another shape has to be contiguous, as the rows."""
    if t is None:
        return None
    shape, strides = lie
    if t.dtype is dtype and t.is_cuda and t.shape == shape and t.stride() == strides:
        return t.data_ptr()
    assert t.is_cuda, "device tensors must be on the GPU"
    # (a dtype of None, sizes below one: a descriptor that is refused, or nothing to read)
    assert t.dtype is dtype or dtype is None, "a tensor has another type than its descriptor"
    if min(shape) >= 1:
        want = [(n, s) for n, s in zip(shape, strides) if n > 1]
        if t.shape == shape:
            assert [(n, s) for n, s in zip(t.shape, t.stride()) if n > 1] == want, "a tensor has other strides than its descriptor"
        else:
            dense, n = [], 1
            for size in reversed(shape):
                dense.append(n)
                n *= size
            assert t.is_contiguous() and t.numel() >= n and want == [(size, s) for size, s in zip(shape, reversed(dense)) if size > 1], \
                "a tensor has another size or strides than its descriptor"
    return t.data_ptr()


def attention_desc(N: int, Lq: int, Lk: int, heads: int, kv_heads: int, D: int, dtype, causal: bool = False, scale: Optional[float] = None,
                   q=(0, 0, 0), k=(0, 0, 0), v=(0, 0, 0), o=(0, 0, 0)):
    """The qrm_attention_desc of queries [N,Lq,heads,D] and keys [N,Lk,kv_heads,D] of `dtype`; scale None is 1 / sqrt(D); q, k, v, o are the strides of
    neighbouring rows, heads and images in elements, 0 = dense."""
    scale = D ** -0.5 if scale is None and D > 0 else 1.0 if scale is None else scale
    return _AttentionDesc(int(N), int(Lq), int(Lk), int(heads), int(kv_heads), int(D), type_code(dtype), int(causal), float(scale),
                          *[int(x) for lie in (q, k, v, o) for x in lie])


def _tensor_addresses():
    """The binding's own module for lists of tensors (csrc/tensors.cpp), which takes what torch's libraries have: torch is imported before it."""
    import torch  # noqa: F401
    try:
        from . import _tensors
    except ImportError as e:
        raise ImportError("_tensors.so is missing or was built for another torch: run `python -m paper_2509_02447_amd.build`") from e
    return _tensors.pointers


def _hptr(t) -> Optional[int]:
    """Host pointer of a CPU torch tensor or a numpy array (or None)."""
    if t is None:
        return None
    if isinstance(t, np.ndarray):
        assert t.flags["C_CONTIGUOUS"], "host arrays must be contiguous"
        return t.ctypes.data
    assert not t.is_cuda and t.is_contiguous(), "host tensors must be contiguous and on the CPU"
    return t.data_ptr()


def _stream_handle(stream) -> Optional[int]:
    if stream is None:
        import torch
        return torch.cuda.current_stream().cuda_stream or None
    if isinstance(stream, int):
        return stream or None
    return stream.cuda_stream or None


class Context:
    """Owns one qrm_ctx.  `weights` is the dict produced by synth.extractor_weights (host fp32 arrays),
    `rs` a dict(m=, prim_poly=, n=, k=, fcr=).  Either may be None."""

    def __init__(self, weights: Optional[dict] = None, rs: Optional[dict] = None, device: int = 0,
                 final_relu: int = 0):
        self._lib = load_library()
        self._h = C.c_void_p()
        ext_p, rs_p = None, None
        keep = []
        if weights is not None:
            d = _ExtDesc()
            d.in_ch, d.n_blocks = int(weights["in_ch"]), int(weights["n_blocks"])
            d.channels, d.n_bits = int(weights["channels"]), int(weights["n_bits"])
            nb, Cc, nbits = d.n_blocks, d.channels, d.n_bits
            arr = {}
            for key in ("conv_w", "scale", "bias", "lin_w", "lin_b"):
                v = weights.get(key)
                arr[key] = None if v is None else np.ascontiguousarray(v, dtype=np.float32)
                keep.append(arr[key])
            expect = Cc * d.in_ch * 9 + (nb - 1) * Cc * Cc * 9 + nbits * Cc * 9
            if arr["conv_w"] is None or arr["conv_w"].size != expect:
                raise ValueError("conv_w has the wrong number of elements")
            d.conv_w, d.scale, d.bias = _fptr(arr["conv_w"]), _fptr(arr["scale"]), _fptr(arr["bias"])
            d.final_affine = int(arr["scale"] is not None and arr["scale"].size == nb * Cc + nbits)
            d.final_relu = int(final_relu)
            d.lin_w, d.lin_b = _fptr(arr["lin_w"]), _fptr(arr["lin_b"])
            for i in range(3):
                d.mean[i] = float(weights["mean"][i])
                d.std[i] = float(weights["std"][i])
            ext_p = C.byref(d)
            self.n_bits, self.channels, self.n_blocks = nbits, Cc, nb
        if rs is not None:
            r = _RsDesc(int(rs["m"]), int(rs["prim_poly"]), int(rs["n"]), int(rs["k"]), int(rs.get("fcr", 1)))
            rs_p = C.byref(r)
            self.n, self.k, self.m = int(rs["n"]), int(rs["k"]), int(rs["m"])
        st = self._lib.qrm_create(ext_p, rs_p, int(device), C.byref(self._h))
        if st != QRM_OK:
            raise QrmError(st, self._lib.qrm_last_error(None).decode())

    # -- plumbing
    def close(self):
        if getattr(self, "_h", None) is not None and self._h:
            self._lib.qrm_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, st: int):
        if st != QRM_OK:
            raise QrmError(st, self._lib.qrm_last_error(self._h).decode())

    def last_error(self) -> str:
        return self._lib.qrm_last_error(self._h).decode()

    # -- the C ABI, one method per entry point
    def qrm_set_micro_batch(self, images: int):
        self._check(self._lib.qrm_set_micro_batch(self._h, int(images)))

    def qrm_profile_enable(self, on: bool):
        self._check(self._lib.qrm_profile_enable(self._h, int(bool(on))))

    def qrm_profile_read(self, kind: int):
        """-> (milliseconds, launches, algorithmic FLOPs) of the timed launches of one kind since enable."""
        ms, n, fl = C.c_double(), C.c_int64(), C.c_double()
        self._check(self._lib.qrm_profile_read(self._h, int(kind), C.byref(ms), C.byref(n), C.byref(fl)))
        return ms.value, n.value, fl.value

    def qrm_profile_read_chunks(self, max_chunks: int):
        """-> float64 array [chunks, 5]: upload start / end, kernels start / end, download end (ms) of the last
        qrm_detect_host call made with profiling on."""
        buf = np.zeros((max(1, int(max_chunks)), 5), dtype=np.float64)
        n = C.c_int32()
        self._check(self._lib.qrm_profile_read_chunks(self._h, int(max_chunks), buf.ctypes.data_as(C.POINTER(C.c_double)),
                                                      C.byref(n)))
        return buf[:min(int(n.value), int(max_chunks))]

    def qrm_release_stream(self, stream=None):
        self._check(self._lib.qrm_release_stream(self._h, _stream_handle(stream)))

    def qrm_diag_set_flags(self, flags: int):
        self._check(self._lib.qrm_diag_set_flags(self._h, int(flags)))

    def qrm_diag_chain_patience(self, looks: int):
        self._check(self._lib.qrm_diag_chain_patience(self._h, int(looks)))

    def qrm_diag_chain_count(self, shared: bool, image: int, value: int, stream=None):
        self._check(self._lib.qrm_diag_chain_count(self._h, _stream_handle(stream), int(bool(shared)), int(image), int(value)))

    def qrm_diag_chain_left_over(self, shared: bool, value: int, stream=None):
        self._check(self._lib.qrm_diag_chain_left_over(self._h, _stream_handle(stream), int(bool(shared)), int(value)))

    def qrm_diag_workspace(self, stream=None):
        """-> (address or None, bytes, earlier ones that are kept) of the workspace of a stream."""
        ws, size, kept = C.c_void_p(), C.c_int64(), C.c_int32()
        self._check(self._lib.qrm_diag_workspace(self._h, _stream_handle(stream), C.byref(ws), C.byref(size), C.byref(kept)))
        return ws.value, size.value, kept.value

    def qrm_diag_matrix_rate(self, data: int) -> float:
        """-> TFLOP/s the matrix pipes sustain on zeros (0), a constant (1) or random operands (2)."""
        v = C.c_double()
        self._check(self._lib.qrm_diag_matrix_rate(self._h, int(data), C.byref(v)))
        return v.value

    def qrm_workspace_bytes(self, N: int, tile_h: int, tile_w: int) -> int:
        return int(self._lib.qrm_workspace_bytes(self._h, int(N), int(tile_h), int(tile_w)))

    def qrm_extract_tiles(self, d_images, N, H, W, d_off_yx, tile, d_tiles, stream=None):
        self._check(self._lib.qrm_extract_tiles(self._h, _dptr(d_images), int(N), int(H), int(W), _dptr(d_off_yx),
                                                int(tile), _dptr(d_tiles), _stream_handle(stream)))

    def qrm_preprocess(self, d_raw, N, H_in, W_in, size, d_off_yx, tile, d_out, stream=None):
        self._check(self._lib.qrm_preprocess(self._h, _dptr(d_raw), int(N), int(H_in), int(W_in), int(size),
                                             _dptr(d_off_yx), int(tile), _dptr(d_out), _stream_handle(stream)))

    def qrm_select_tiles_variance(self, d_images, N, H, W, tile, stride, d_off_yx, d_scores=None, stream=None):
        self._check(self._lib.qrm_select_tiles_variance(self._h, _dptr(d_images), int(N), int(H), int(W), int(tile),
                                                        int(stride), _dptr(d_off_yx), _dptr(d_scores),
                                                        _stream_handle(stream)))

    def qrm_extractor_forward(self, d_tiles, N, h, w, d_logits, d_bits=None, stream=None):
        self._check(self._lib.qrm_extractor_forward(self._h, _dptr(d_tiles), int(N), int(h), int(w), _dptr(d_logits),
                                                    _dptr(d_bits), _stream_handle(stream)))

    def qrm_extractor_blocks(self, d_tiles, N, h, w, n_run, d_act, stream=None):
        self._check(self._lib.qrm_extractor_blocks(self._h, _dptr(d_tiles), int(N), int(h), int(w), int(n_run),
                                                   _dptr(d_act), _stream_handle(stream)))

    def qrm_rs_decode(self, d_symbols, N, d_msg, d_codeword, d_nerr, stream=None):
        self._check(self._lib.qrm_rs_decode(self._h, _dptr(d_symbols), int(N), _dptr(d_msg), _dptr(d_codeword),
                                            _dptr(d_nerr), _stream_handle(stream)))

    def qrm_detect(self, d_images, N, H, W, d_off_yx, tile, d_logits, d_bits, d_msg, d_codeword, d_nerr,
                   stream=None):
        self._check(self._lib.qrm_detect(self._h, _dptr(d_images), int(N), int(H), int(W), _dptr(d_off_yx),
                                         int(tile), _dptr(d_logits), _dptr(d_bits), _dptr(d_msg), _dptr(d_codeword),
                                         _dptr(d_nerr), _stream_handle(stream)))

    def qrm_detect_static(self, d_images, N, H, W, d_off_yx, tile, d_logits, d_bits, d_msg, d_codeword, d_nerr,
                          stream=None):
        self._check(self._lib.qrm_detect_static(self._h, _dptr(d_images), int(N), int(H), int(W), _dptr(d_off_yx),
                                                int(tile), _dptr(d_logits), _dptr(d_bits), _dptr(d_msg),
                                                _dptr(d_codeword), _dptr(d_nerr), _stream_handle(stream)))

    def qrm_detect_host(self, h_chunks, chunk_images, H, W, h_off_chunks, tile, depth, h_msg, h_codeword, h_nerr):
        """h_chunks / h_off_chunks: sequences of host buffers (pinned CPU tensors or numpy arrays), one per chunk."""
        n = len(h_chunks)
        chunks = (C.c_void_p * max(1, n))(*[_hptr(t) for t in h_chunks])
        offs = None
        if h_off_chunks is not None:
            assert len(h_off_chunks) == n
            offs = (C.c_void_p * max(1, n))(*[_hptr(t) for t in h_off_chunks])
        self._check(self._lib.qrm_detect_host(self._h, chunks, int(n), int(chunk_images), int(H), int(W), offs, int(tile),
                                              int(depth), _hptr(h_msg), _hptr(h_codeword), _hptr(h_nerr)))

    def qrm_set_key(self, h_key, tau: int):
        key = np.ascontiguousarray(h_key, dtype=np.uint8).reshape(-1)
        assert key.size == self.k, "the key has k symbols"
        self._check(self._lib.qrm_set_key(self._h, key.ctypes.data, int(tau)))

    def qrm_verify_key(self, d_msg, N, d_matches, d_detected=None, stream=None):
        self._check(self._lib.qrm_verify_key(self._h, _dptr(d_msg), int(N), _dptr(d_matches), _dptr(d_detected),
                                             _stream_handle(stream)))

    def qrm_detect_verify(self, d_images, N, H, W, d_off_yx, tile, d_logits, d_bits, d_msg, d_codeword, d_nerr,
                          d_matches, d_detected=None, stream=None):
        self._check(self._lib.qrm_detect_verify(self._h, _dptr(d_images), int(N), int(H), int(W), _dptr(d_off_yx),
                                                int(tile), _dptr(d_logits), _dptr(d_bits), _dptr(d_msg),
                                                _dptr(d_codeword), _dptr(d_nerr), _dptr(d_matches), _dptr(d_detected),
                                                _stream_handle(stream)))

    def qrm_group_norm(self, desc, d_x, d_gamma, d_beta, d_y, d_mean=None, d_rstd=None, stream=None):
        dtype, shape, x, y, stats = desc.maps()
        f32, C_ = _kinds().f32, shape[2]
        self._check(self._lib.qrm_group_norm(self._h, C.byref(desc), _dptr_map(d_x, dtype, shape, x), _dptr_of(d_gamma, f32, C_),
                                             _dptr_of(d_beta, f32, C_), _dptr_map(d_y, dtype, shape, y), _dptr_of(d_mean, f32, stats),
                                             _dptr_of(d_rstd, f32, stats), _stream_handle(stream)))

    def qrm_group_norm_backward(self, desc, d_x, d_dy, d_gamma, d_beta, d_mean, d_rstd, d_dx, d_dgamma=None, d_dbeta=None,
                                stream=None):
        dtype, shape, x, y, stats = desc.maps()
        f32, C_ = _kinds().f32, shape[2]
        self._check(self._lib.qrm_group_norm_backward(self._h, C.byref(desc), _dptr_map(d_x, dtype, shape, x), _dptr_map(d_dy, dtype, shape, y),
                                                      _dptr_of(d_gamma, f32, C_), _dptr_of(d_beta, f32, C_), _dptr_of(d_mean, f32, stats),
                                                      _dptr_of(d_rstd, f32, stats), _dptr_map(d_dx, dtype, shape, x), _dptr_of(d_dgamma, f32, C_),
                                                      _dptr_of(d_dbeta, f32, C_), _stream_handle(stream)))

    def qrm_attention(self, desc, d_q, d_k, d_v, d_o, d_lse=None, d_q_len=None, d_k_len=None, stream=None):
        dtype, lie, sums = desc.rows()
        k, N = _kinds(), desc.N
        self._check(self._lib.qrm_attention(self._h, C.byref(desc), _dptr_rows(d_q, dtype, lie["q"]), _dptr_rows(d_k, dtype, lie["k"]),
                                            _dptr_rows(d_v, dtype, lie["v"]), _dptr_of(d_q_len, k.i32, N), _dptr_of(d_k_len, k.i32, N),
                                            _dptr_rows(d_o, dtype, lie["o"]), _dptr_of(d_lse, k.f32, sums), _stream_handle(stream)))

    def qrm_attention_backward(self, desc, d_q, d_k, d_v, d_o, d_do, d_lse, d_dq, d_dk=None, d_dv=None, d_q_len=None, d_k_len=None, stream=None):
        dtype, lie, sums = desc.rows()
        k, N = _kinds(), desc.N
        rows = lambda t, name: _dptr_rows(t, dtype, lie[name])
        self._check(self._lib.qrm_attention_backward(self._h, C.byref(desc), rows(d_q, "q"), rows(d_k, "k"), rows(d_v, "v"), rows(d_o, "o"), rows(d_do, "o"),
                                                     _dptr_of(d_lse, k.f32, sums), _dptr_of(d_q_len, k.i32, N), _dptr_of(d_k_len, k.i32, N),
                                                     rows(d_dq, "q"), rows(d_dk, "k"), rows(d_dv, "v"), _stream_handle(stream)))

    def qrm_unpack_moment(self, moment: int, d_codes, d_scales, n, d_out, stream=None):
        n = int(n)
        code = type_code(d_out.dtype)
        self._check(self._lib.qrm_unpack_moment(self._h, int(moment), _dptr_bytes(d_codes, n), _dptr_of(d_scales, _kinds().f32, -(-n // QRM_MOMENT_BLOCK)),
                                                n, code, _dptr_of(d_out, d_out.dtype, n), _stream_handle(stream)))

    def qrm_message_loss(self, d_logits, d_target, target_rows, N, n_bits, rs_weight, d_loss, d_grad=None, d_bit_errors=None,
                         d_symbol_errors=None, stream=None):
        N, n_bits, target_rows = int(N), int(n_bits), int(target_rows)
        k, cells = _kinds(), N * n_bits
        f32, i32 = k.f32, k.i32
        self._check(self._lib.qrm_message_loss(self._h, _dptr_of(d_logits, f32, cells), _dptr_bytes(d_target, target_rows * n_bits), target_rows,
                                               N, n_bits, float(rs_weight), _dptr_of(d_loss, f32, 1), _dptr_of(d_grad, f32, cells),
                                               _dptr_of(d_bit_errors, i32, N), _dptr_of(d_symbol_errors, i32, N), _stream_handle(stream)))


class AdamW:
    """Owns one qrm_adamw.  `tensors`: a list of dict(param=, m=, v=, and as needed m_scale=, v_scale=, copy=, weight_decay=0.0,
    lr_scale=1.0) of device tensors, all parameters of one type; moments are f32, or int8 (m) and uint8 (v) codes with f32 scales,
    one for QRM_MOMENT_BLOCK elements.  The object keeps the tensors alive, and `ctx`, which reports its errors."""

    def __init__(self, ctx: Context, tensors, grad_type):
        self._h = C.c_void_p()
        self._ctx, self._keep = ctx, [dict(t) for t in tensors]
        self._lib = ctx._lib
        n = len(self._keep)
        rows = (_AdamwTensor * max(1, n))()
        for r, t in zip(rows, self._keep):
            self._check_sizes(t)
            r.n = t["param"].numel()
            r.d_param, r.d_m, r.d_v = _dptr(t["param"]), _dptr(t["m"]), _dptr(t["v"])
            r.d_m_scale, r.d_v_scale, r.d_copy = _dptr(t.get("m_scale")), _dptr(t.get("v_scale")), _dptr(t.get("copy"))
            r.weight_decay, r.lr_scale = float(t.get("weight_decay", 0.0)), float(t.get("lr_scale", 1.0))
        one = lambda types, what: (types.pop() if len(types) == 1 else self._mixed(what)) if types else None
        import torch
        param = one({t["param"].dtype for t in self._keep}, "parameters") or torch.float32
        moment = one({t["m"].dtype for t in self._keep}, "moments") or torch.float32
        copy = one({t["copy"].dtype for t in self._keep if t.get("copy") is not None}, "copies")
        desc = _AdamwDesc(n, type_code(param), type_code(grad_type), QRM_BF16 if copy is None else type_code(copy),
                          {torch.float32: 32, torch.int8: 8}[moment])
        ctx._check(self._lib.qrm_adamw_create(ctx._h, C.byref(desc), rows, C.byref(self._h)))
        self._grad_type, self._sizes = grad_type, (C.c_int64 * n)(*[t["param"].numel() for t in self._keep])
        self._array, self._addresses = C.c_void_p * max(1, n), _tensor_addresses()

    @staticmethod
    def _check_sizes(t):
        import torch
        n, eight = t["param"].numel(), t["m"].dtype == torch.int8
        assert t["m"].numel() == n and t["v"].numel() == n, "moments have their parameters' sizes"
        assert t["v"].dtype == (torch.uint8 if eight else t["m"].dtype), "moments are f32 both, or int8 and uint8"
        if eight and n:
            assert all(t[k].dtype == torch.float32 and t[k].numel() == -(-n // QRM_MOMENT_BLOCK) for k in ("m_scale", "v_scale")), \
                "8-bit moments have one f32 scale for QRM_MOMENT_BLOCK elements"
        assert t.get("copy") is None or t["copy"].numel() == n, "a copy has its parameters' size"

    @staticmethod
    def _mixed(what):
        raise ValueError(f"all {what} of a plan have one type")

    def _pointers(self, grads):
        return self._array.from_buffer(self._addresses(grads, self._sizes, self._grad_type))

    def qrm_adamw_grad_norm(self, grads, max_norm: float, d_norm, d_scale, d_unscale=None, stream=None):
        """grads as in qrm_adamw_step; d_norm, d_scale, d_unscale: f32 [1] on the device (or None)."""
        f32 = _kinds().f32
        self._ctx._check(self._lib.qrm_adamw_grad_norm(self._ctx._h, self._h, self._pointers(grads), float(max_norm), _dptr_of(d_unscale, f32, 1),
                                                       _dptr_of(d_norm, f32, 1), _dptr_of(d_scale, f32, 1), _stream_handle(stream)))

    def qrm_adamw_scale_grads(self, grads, d_scale, outs=None, stream=None):
        """outs: a tensor for each gradient, or None: in place."""
        ptrs = self._pointers(grads)
        self._ctx._check(self._lib.qrm_adamw_scale_grads(self._ctx._h, self._h, ptrs, _dptr_of(d_scale, _kinds().f32, 1),
                                                         ptrs if outs is None else self._pointers(outs), _stream_handle(stream)))

    def qrm_adamw_step(self, grads, step: int, lr: float, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8,
                       d_grad_scale=None, stream=None):
        """grads: one device tensor of grad_type for each tensor of the plan, or None where it has no gradient."""
        ptrs = self._pointers(grads)
        self._ctx._check(self._lib.qrm_adamw_step(self._ctx._h, self._h, ptrs, int(step), float(lr), float(beta1), float(beta2),
                                                  float(eps), _dptr_of(d_grad_scale, _kinds().f32, 1), _stream_handle(stream)))

    def close(self):
        if getattr(self, "_h", None) is not None and self._h:
            self._lib.qrm_adamw_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
