"""ctypes declarations of the C ABI in ``include/hpacml.h`` (argument
marshalling only: every step of the region runs in the HIP library)."""
from __future__ import annotations

import ctypes as C
import os

MAX_RANK = 4
OK, E_INVAL, E_SHAPE, E_RANGE, E_ALIAS, E_UNSUPPORTED, E_NOMEM, E_DEVICE = range(8)
TO, FROM = 0, 1
BND_NONE, BND_PERIODIC, BND_CLAMP = 0, 1, 2
F32, BF16 = 0, 1
ACT_IDENTITY, ACT_RELU = 0, 1
LAYER_CONV2D, LAYER_MAXPOOL2D, LAYER_LINEAR = 0, 1, 2
MODE_INFER, MODE_COLLECT, MODE_PREDICATED = 0, 1, 2
PAD_VALID, PAD_SAME = 0, 1
PADMODE_ZEROS, PADMODE_CIRCULAR, PADMODE_REPLICATE = 0, 1, 2

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libhpacml.so")


class Slice(C.Structure):
    _fields_ = [("lo", C.c_int32 * MAX_RANK), ("count", C.c_int32 * MAX_RANK)]


class Functor(C.Structure):
    _fields_ = [("rank", C.c_int32), ("n_slices", C.c_int32),
                ("slices", C.POINTER(Slice)), ("n_features", C.c_int32)]


class Array(C.Structure):
    _fields_ = [("data", C.c_void_p), ("dtype", C.c_int32), ("reserved", C.c_int32),
                ("extent", C.c_int64 * MAX_RANK), ("stride", C.c_int64 * MAX_RANK)]


class Sweep(C.Structure):
    _fields_ = [("start", C.c_int64 * MAX_RANK), ("stop", C.c_int64 * MAX_RANK),
                ("step", C.c_int64 * MAX_RANK)]


class Checkpoint8(C.Structure):
    """``hpacml8_checkpoint``"""
    _fields_ = [("codes", C.c_void_p), ("exps", C.c_void_p), ("rows", C.c_int64), ("ld_codes", C.c_int64),
                ("ld_exps", C.c_int64), ("width", C.c_int32), ("act", C.c_int32)]


class Matrix(C.Structure):
    """``hpacmlt_matrix``"""
    _fields_ = [("codes", C.c_void_p), ("scales", C.c_void_p), ("rows", C.c_int64), ("width", C.c_int64)]


class Gradient(C.Structure):
    """``hpacmlt_gradient``"""
    _fields_ = [("from_", C.c_void_p), ("to", C.c_void_p), ("count", C.c_int64), ("from_dtype", C.c_int32),
                ("to_dtype", C.c_int32)]


class Layer(C.Structure):
    _fields_ = [("kind", C.c_int32), ("out_channels", C.c_int32), ("kernel", C.c_int32 * 2),
                ("stride", C.c_int32 * 2), ("padding", C.c_int32), ("pad_mode", C.c_int32), ("act", C.c_int32)]


# hpacml_accurate_fn: void (*)(void *user, void *stream)
ACCURATE_FN = C.CFUNCTYPE(None, C.c_void_p, C.c_void_p)

# every symbol the header declares, with (restype, argtypes)
_P = C.POINTER
SIGNATURES = {
    "hpacml_abi_version": (C.c_int32, []),
    "hpacml_status_string": (C.c_char_p, [C.c_int]),
    "hpacml_map_validate": (C.c_int, [_P(Functor), C.c_int32, _P(Array), C.c_int32, _P(Sweep),
                                      _P(C.c_int32), _P(C.c_int64), _P(C.c_int32)]),
    "hpacml_map_create": (C.c_int, [_P(Functor), C.c_int32, _P(Array), C.c_int32, _P(Sweep),
                                    _P(C.c_int32), _P(C.c_void_p)]),
    "hpacml_map_shape": (C.c_int, [C.c_void_p, _P(C.c_int64), _P(C.c_int32)]),
    "hpacml_map_destroy": (None, [C.c_void_p]),
    "hpacml_model_validate": (C.c_int, [C.c_int32, _P(C.c_int32), _P(C.c_int32), C.c_int32]),
    "hpacml_model_create": (C.c_int, [C.c_int32, _P(C.c_int32), _P(_P(C.c_float)), _P(_P(C.c_float)),
                                      _P(C.c_int32), C.c_int32, _P(C.c_void_p)]),
    "hpacml_model_destroy": (None, [C.c_void_p]),
    "hpacml_infer": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]),
    "hpacml_infer_noalloc": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]),
    "hpacml_collect": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p]),
    "hpacml_collect_pair": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p, C.c_int64,
                                      C.c_void_p]),
    "hpacml_infer_variant": (C.c_char_p, [C.c_void_p, C.c_void_p, C.c_void_p]),
    "hpacml_cnn_validate": (C.c_int, [C.c_int32, C.c_int32, C.c_int32, C.c_int32, _P(Layer), _P(C.c_int32)]),
    "hpacml_cnn_param_counts": (C.c_int, [C.c_int32, C.c_int32, C.c_int32, C.c_int32, _P(Layer), _P(C.c_int64),
                                          _P(C.c_int64)]),
    "hpacml_cnn_create": (C.c_int, [C.c_int32, C.c_int32, C.c_int32, C.c_int32, _P(Layer), _P(_P(C.c_float)),
                                    _P(_P(C.c_float)), C.c_int32, _P(C.c_void_p)]),
    "hpacml_region_create": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int64,
                                       _P(C.c_void_p)]),
    "hpacml_region_run": (C.c_int, [C.c_void_p, C.c_int32, C.c_int32, ACCURATE_FN, C.c_void_p, C.c_void_p]),
    "hpacml_region_samples": (C.c_int, [C.c_void_p, _P(C.c_int64)]),
    "hpacml_region_read": (C.c_int, [C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p, C.c_void_p]),
    "hpacml_region_save": (C.c_int, [C.c_void_p, C.c_char_p, C.c_char_p]),
    "hpacml_region_reset": (C.c_int, [C.c_void_p]),
    "hpacml_region_destroy": (None, [C.c_void_p]),
}

# every symbol of include/hpacml8.h (dense layers in 8 bits)
BLOCK8, MAX_WIDTH8 = 32, 16384
SIGNATURES8 = {
    "hpacml8_linear_create": (C.c_int, [C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, _P(C.c_void_p)]),
    "hpacml8_linear_destroy": (None, [C.c_void_p]),
    "hpacml8_linear_scratch": (C.c_int, [C.c_void_p, C.c_int64, _P(C.c_size_t)]),
    "hpacml8_linear_run": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int32, C.c_int64, C.c_int64, C.c_void_p, C.c_int32,
                                     C.c_int64, C.c_int32, C.c_void_p, C.c_size_t, C.c_void_p]),
    "hpacml8_checkpoint_save": (C.c_int, [_P(Checkpoint8), C.c_void_p, C.c_int32, C.c_int64, C.c_void_p, C.c_int32,
                                          C.c_int64, C.c_void_p]),
    "hpacml8_checkpoint_load": (C.c_int, [_P(Checkpoint8), C.c_void_p, C.c_int32, C.c_int64, C.c_void_p]),
    "hpacml8_backward_scratch": (C.c_int, [_P(Checkpoint8), C.c_void_p, C.c_int32, C.c_int64, C.c_int32, C.c_int32,
                                           C.c_int32, _P(C.c_size_t)]),
    "hpacml8_backward": (C.c_int, [_P(Checkpoint8), C.c_void_p, C.c_int32, C.c_int64, C.c_int32, C.c_void_p, C.c_int64,
                                   C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p, C.c_int64, C.c_int32, C.c_void_p,
                                   C.c_size_t, C.c_void_p]),
}

# every symbol of include/hpacmlt.h (layers in 8-bit floating point, group norm, gradients)
ACT_SILU = 2
NORM_2, NORM_MAX = 0, 1
BLOCKF8, MAX_CHANNELS = 128, 16384
_GN = [C.c_void_p, C.c_int32, C.c_int64, C.c_int64, C.c_int64, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p]
SIGNATURES_T = {
    "hpacmlt_matrix_bytes": (C.c_int, [C.c_int64, C.c_int64, _P(C.c_size_t), _P(C.c_size_t)]),
    "hpacmlt_quantize": (C.c_int, [C.c_void_p, C.c_int32, C.c_int64, C.c_int64, C.c_int64, _P(Matrix), _P(Matrix), C.c_int32,
                                   C.c_void_p]),
    "hpacmlt_load": (C.c_int, [_P(Matrix), C.c_void_p, C.c_int32, C.c_int64, C.c_void_p]),
    "hpacmlt_product": (C.c_int, [_P(Matrix), _P(Matrix), C.c_void_p, C.c_int32, C.c_void_p, C.c_int32, C.c_int64, C.c_int32,
                                  C.c_void_p, C.c_size_t, C.c_void_p]),
    "hpacmlt_product_scratch": (C.c_int, [C.c_int64, C.c_int64, C.c_int64, _P(C.c_size_t)]),
    "hpacmlt_linear_run": (C.c_int, [_P(Matrix), C.c_void_p, C.c_void_p, C.c_int32, C.c_int64, C.c_int64, C.c_void_p, C.c_int32,
                                     C.c_int64, C.c_int32, _P(Matrix), C.c_void_p, C.c_size_t, C.c_void_p]),
    "hpacmlt_linear_scratch": (C.c_int, [_P(Matrix), C.c_int64, _P(C.c_size_t)]),
    "hpacmlt_backward": (C.c_int, [_P(Matrix), C.c_void_p, C.c_void_p, C.c_int32, C.c_int64, C.c_int64, C.c_int32, _P(Matrix),
                                   C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p, C.c_int64, C.c_int32, C.c_void_p, C.c_size_t,
                                   C.c_void_p]),
    "hpacmlt_backward_scratch": (C.c_int, [C.c_int64, C.c_int64, C.c_int32, C.c_int32, C.c_int32, C.c_int32, _P(C.c_size_t)]),
    "hpacmlt_group_norm": (C.c_int, _GN + [C.c_float, C.c_int32, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p, C.c_void_p,
                                           C.c_size_t, C.c_void_p]),
    "hpacmlt_group_norm_backward": (C.c_int, _GN + [C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64,
                                                    C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_size_t, C.c_void_p]),
    "hpacmlt_group_norm_scratch": (C.c_int, [C.c_int32, C.c_int64, C.c_int64, C.c_int32, C.c_int32, C.c_int32, _P(C.c_size_t)]),
    "hpacmlt_gradients_create": (C.c_int, [_P(Gradient), C.c_int64, _P(C.c_void_p)]),
    "hpacmlt_gradients_destroy": (None, [C.c_void_p]),
    "hpacmlt_gradients_scratch": (C.c_int, [C.c_void_p, _P(C.c_size_t)]),
    "hpacmlt_gradients_norm": (C.c_int, [C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "hpacmlt_gradients_clip": (C.c_int, [C.c_void_p, C.c_int32, C.c_double, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
}

_lib = None


def lib():
    """Load the built library; raise if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("libhpacml.so is not built: run `python -m paper_2407_18352_amd.build` "
                               "(or __graft_entry__.build())")
        L = C.CDLL(LIB_PATH)
        for name, (res, args) in [*SIGNATURES.items(), *SIGNATURES8.items(), *SIGNATURES_T.items()]:
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _lib = L
    return _lib


class HpacmlError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        msg = lib().hpacml_status_string(status).decode()
        super().__init__("%s failed: %s (status %d)" % (what, msg, status))


def check(status: int, what: str) -> None:
    if status != OK:
        raise HpacmlError(status, what)
