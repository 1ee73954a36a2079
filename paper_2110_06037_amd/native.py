"""ctypes binding of libsoftneuro.so (the C ABI in include/softneuro.h).

Argument marshalling only: every step of the path runs inside the library.
The library is loaded from this package directory; if it is missing the
import fails loudly (there is no fallback implementation).
"""

from __future__ import annotations

import ctypes
import os

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libsoftneuro.so")

# enums of softneuro.h
F32, F16, BF16 = 0, 1, 2
DTYPE = {"f32": F32, "f16": F16, "bf16": BF16}
NCHW, NHWC, NC8HW8 = 0, 1, 2
LAYOUT = {"NCHW": NCHW, "NHWC": NHWC, "NC8HW8": NC8HW8}
LAYOUT_NAME = {v: k for k, v in LAYOUT.items()}
DIRECT, IGEMM, WINOGRAD = 0, 1, 2
ALGO = {"direct": DIRECT, "igemm": IGEMM, "winograd": WINOGRAD}
ALGO_NAME = {v: k for k, v in ALGO.items()}
L_INPUT, L_CONV2D, L_MAXPOOL, L_GAP, L_ADD, L_FC, L_OUTPUT = range(7)
ACT = {"none": 0, "relu": 1, "relu6": 2}
SELECT_DPRS, SELECT_FIXED = 0, 1
OPT_LAYOUTS, OPT_ALGOS, OPT_PARAMS, OPT_HIPGRAPH, OPT_SEED, OPT_FLUSH, OPT_KEEP, OPT_DTYPES, OPT_WS_LIMIT = range(9)
DTYPE_NAME = {v: k for k, v in DTYPE.items()}
NORM = {"rms": 0, "layer": 1}
GATE = {"none": 0, "before": 1, "after": 2}
PAIRS = {"halves": 0, "neighbours": 1}
STORE = {"same": 0, "i8": 1}

STATUS = {0: "SN_OK", -1: "SN_E_INVALID", -2: "SN_E_SHAPE", -3: "SN_E_STATE",
          -4: "SN_E_UNSUPPORTED", -5: "SN_E_DEVICE", -6: "SN_E_NOMEM", -7: "SN_E_INTERNAL"}


class SNError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"{STATUS.get(code, code)}: {msg}")
        self.code = code


class LayerDesc(ctypes.Structure):
    _fields_ = [("type", ctypes.c_int32), ("k", ctypes.c_int32), ("r", ctypes.c_int32),
                ("s", ctypes.c_int32), ("stride", ctypes.c_int32), ("pad", ctypes.c_int32),
                ("groups", ctypes.c_int32), ("act", ctypes.c_int32)]


class RoutineDesc(ctypes.Structure):
    _fields_ = [("id", ctypes.c_int32), ("layout", ctypes.c_int32), ("algo", ctypes.c_int32),
                ("param", ctypes.c_int32), ("dtype", ctypes.c_int32), ("schema", ctypes.c_int32),
                ("cost_ns", ctypes.c_int64), ("ws_bytes", ctypes.c_int64), ("name", ctypes.c_char * 64)]


class NormDesc(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("res_dtype", ctypes.c_int32), ("dim", ctypes.c_int32),
                ("groups", ctypes.c_int32), ("kind", ctypes.c_int32), ("gate", ctypes.c_int32),
                ("eps", ctypes.c_float), ("scale", ctypes.c_float)]


class Linear4Desc(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("rows", ctypes.c_int32), ("cols", ctypes.c_int32),
                ("group", ctypes.c_int32), ("act", ctypes.c_int32)]


class ScanDesc(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("groups", ctypes.c_int32), ("state", ctypes.c_int32), ("conv", ctypes.c_int32),
                ("max_seqs", ctypes.c_int32), ("max_tokens", ctypes.c_int64)]


class ScanIO(ctypes.Structure):
    _fields_ = [("seqs", ctypes.c_int32), ("tokens", ctypes.c_int64), ("offsets", ctypes.c_void_p),
                ("x", ctypes.c_void_p), ("x_stride", ctypes.c_int64), ("dt", ctypes.c_void_p),
                ("dt_stride", ctypes.c_int64), ("window", ctypes.c_void_p), ("state", ctypes.c_void_p),
                ("y", ctypes.c_void_p), ("y_stride", ctypes.c_int64), ("window_out", ctypes.c_void_p),
                ("state_out", ctypes.c_void_p)]


class HeadNormDesc(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("heads", ctypes.c_int32), ("kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("rot", ctypes.c_int32), ("pairs", ctypes.c_int32),
                ("norm", ctypes.c_int32), ("eps", ctypes.c_float)]


class CacheDesc(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("store", ctypes.c_int32), ("kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("page", ctypes.c_int32)]


class CacheIO(ctypes.Structure):
    _fields_ = [("pages", ctypes.c_int64), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p), ("seqs", ctypes.c_int32),
                ("width", ctypes.c_int32), ("table", ctypes.c_void_p), ("table_stride", ctypes.c_int64),
                ("past", ctypes.c_void_p), ("tokens", ctypes.c_int64), ("offsets", ctypes.c_void_p)]


class AttnDesc(ctypes.Structure):
    _fields_ = [("cache", CacheDesc), ("heads", ctypes.c_int32), ("window", ctypes.c_int32),
                ("scale", ctypes.c_float), ("max_seqs", ctypes.c_int32), ("max_tokens", ctypes.c_int64)]


# exported functions: name -> (restype, argtypes)
_P = ctypes.c_void_p
_I32 = ctypes.c_int32
_I32P = ctypes.POINTER(ctypes.c_int32)
_I64P = ctypes.POINTER(ctypes.c_int64)
_I64 = ctypes.c_int64
_F32P = ctypes.POINTER(ctypes.c_float)
SIGNATURES = {
    "sn_graph_create": (ctypes.c_int, [_I32, _I32, _I32, _I32, _I32, _I32, ctypes.POINTER(_P)]),
    "sn_set_option": (ctypes.c_int, [_P, _I32, ctypes.c_int64]),
    "sn_add_layer": (ctypes.c_int, [_P, ctypes.POINTER(LayerDesc), _I32P, _I32, _P,
                                    ctypes.POINTER(ctypes.c_float), _I32P]),
    "sn_add_input": (ctypes.c_int, [_P, _I32, _I32, _I32, _I32P]),
    "sn_add_projected_conv": (ctypes.c_int, [_P, ctypes.POINTER(LayerDesc), _I32, _I32, _I32, _P,
                                             ctypes.POINTER(ctypes.c_float), _P, ctypes.POINTER(ctypes.c_float),
                                             _I32P]),
    "sn_mark_output": (ctypes.c_int, [_P, _I32]),
    "sn_num_io": (ctypes.c_int, [_P, _I32P, _I32P]),
    "sn_run_mimo": (ctypes.c_int, [_P, ctypes.POINTER(_P), _I32, ctypes.POINTER(_P), _I32, _P]),
    "sn_profile": (ctypes.c_int, [_P, _I32, _I32, _P]),
    "sn_select_path": (ctypes.c_int, [_P, _I32, _I32, _I32]),
    "sn_set_path": (ctypes.c_int, [_P, _I32P, _I32]),
    "sn_run": (ctypes.c_int, [_P, _P, _P, _P]),
    "sn_run_noalloc": (ctypes.c_int, [_P, _P, _P, _P]),
    "sn_run_timed": (ctypes.c_int, [_P, _P, _P, _P, _I32, ctypes.POINTER(ctypes.c_float), _I32]),
    "sn_layer_output": (ctypes.c_int, [_P, _I32, _P, ctypes.c_size_t, ctypes.POINTER(ctypes.c_size_t),
                                       _I32P, _P]),
    "sn_plan_launches": (ctypes.c_int, [_P, _I32P, _I32, _I32P]),
    "sn_profile_integrated": (ctypes.c_int, [_P, _I32, _I32, _P, _I32P]),
    "sn_integrated_candidate": (ctypes.c_int, [_P, _I32, _I32P, _I32, _I64P, _I64P, _I32P]),
    "sn_refine_in_path": (ctypes.c_int, [_P, _I32, _I32, _I32, _P, _I32P]),
    "sn_get_costs": (ctypes.c_int, [_P, ctypes.c_char_p, ctypes.c_size_t,
                                    ctypes.POINTER(ctypes.c_size_t)]),
    "sn_set_costs": (ctypes.c_int, [_P, ctypes.c_char_p]),
    "sn_get_path": (ctypes.c_int, [_P, _I32P, _I32, _I64P]),
    "sn_num_layers": (ctypes.c_int, [_P, _I32P]),
    "sn_num_routines": (ctypes.c_int, [_P, _I32, _I32P]),
    "sn_routine_info": (ctypes.c_int, [_P, _I32, _I32, ctypes.POINTER(RoutineDesc)]),
    "sn_layer_shape": (ctypes.c_int, [_P, _I32, _I32P]),
    "sn_dp_stats": (ctypes.c_int, [_P, _I32, _I64P, _I64P]),
    "sn_graph_destroy": (None, [_P]),
    "sn_op_destroy": (None, [_P]),
    "sn_norm_create": (ctypes.c_int, [ctypes.POINTER(NormDesc), _F32P, _F32P, _F32P, _F32P, _F32P, _I32,
                                      ctypes.POINTER(_P)]),
    "sn_norm_run": (ctypes.c_int, [_P, _I64, _P, _I64, _P, _I64, _P, _I64, _P, _I64, _P, _I64, _P]),
    "sn_qlinear_create": (ctypes.c_int, [ctypes.POINTER(Linear4Desc), _P, _P, _P, _F32P, _I32, ctypes.POINTER(_P)]),
    "sn_qlinear_run": (ctypes.c_int, [_P, _I64, _P, _I64, _P, _I64, _P]),
    "sn_scan_create": (ctypes.c_int, [ctypes.POINTER(ScanDesc), _F32P, _F32P, _F32P, _F32P, _F32P, _I32,
                                      ctypes.POINTER(_P)]),
    "sn_scan_run": (ctypes.c_int, [_P, ctypes.POINTER(ScanIO), _P]),
    "sn_scan_step": (ctypes.c_int, [_P, ctypes.POINTER(ScanIO), _P]),
    "sn_headnorm_create": (ctypes.c_int, [ctypes.POINTER(HeadNormDesc), _F32P, _F32P, _P, _I32, ctypes.POINTER(_P)]),
    "sn_headnorm_run": (ctypes.c_int, [_P, _I64, _P, _P, _I64, _P, _I64, _P, _I64, _P, _I64, _P]),
    "sn_cache_create": (ctypes.c_int, [ctypes.POINTER(CacheDesc), _I32, ctypes.POINTER(_P)]),
    "sn_cache_write": (ctypes.c_int, [_P, ctypes.POINTER(CacheIO), _P, _I64, _P, _I64, _P]),
    "sn_cache_read": (ctypes.c_int, [_P, ctypes.POINTER(CacheIO), _P, _I64, _P, _I64, _P]),
    "sn_attn_create": (ctypes.c_int, [ctypes.POINTER(AttnDesc), _I32, ctypes.POINTER(_P)]),
    "sn_attn_run": (ctypes.c_int, [_P, ctypes.POINTER(CacheIO), _P, _I64, _P, _I64, _P]),
    "sn_attn_step": (ctypes.c_int, [_P, ctypes.POINTER(CacheIO), _P, _I64, _P, _I64, _P]),
    "sn_last_error": (ctypes.c_char_p, []),
}

_lib = None


def lib():
    """Load the library (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: run paper_2110_06037_amd/build.py "
                              "(or __graft_entry__.build()) first")
        # torch (device memory and streams) must load its HIP runtime first:
        # loaded after the library it would bind to the runtime the library
        # pulled in and find no GPU; loaded before, both share one device view
        import torch  # noqa: F401
        L = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            f = getattr(L, name)
            f.restype = res
            f.argtypes = args
        _lib = L
    return _lib


def check(rc):
    if rc != 0:
        msg = lib().sn_last_error()
        raise SNError(rc, msg.decode() if msg else "")
    return rc
