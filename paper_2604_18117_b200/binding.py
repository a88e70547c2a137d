"""ctypes binding of liblq.so: the same entry points as include/lq.h, argument marshalling only.

Every step of the path runs inside the library's CUDA kernels; PyTorch appears only as the
owner of device buffers and streams.  If the shared library is missing the import of any entry
point raises - there is no CPU fallback.
"""
from __future__ import annotations

import ctypes as C
import os
import struct

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liblq.so")

LQ_OK = 0
BRANCH = {"none": 0, "w16a16": 1, "w8a8": 2, "w6a6": 3, "w4a8": 4, "mxfp8": 5, "mxfp6": 6, "mxfp4": 7,
          "mxint8": 8, "mxint4": 9}
MAIN_AUTO, MAIN_MXFP4, MAIN_MXINT4_A8 = 0, 2, 3
ACT_DEFAULT, ACT_MXFP6 = 0, 6
BRANCH_NAME = {v: k for k, v in BRANCH.items()}
OUT_F16, OUT_F32 = 0, 1
NORM_NONE, NORM_RMS, NORM_LAYER = 0, 1, 2
GROUP = 64


class LqConfig(C.Structure):
    _fields_ = [("K", C.c_int32), ("N", C.c_int32), ("rank", C.c_int32), ("group", C.c_int32),
                ("branch", C.c_int32), ("steps", C.c_int32), ("lr", C.c_float), ("beta1", C.c_float),
                ("beta2", C.c_float), ("eps", C.c_float), ("rot_steps", C.c_int32), ("rot_lr", C.c_float),
                ("seed", C.c_uint64), ("main_fmt", C.c_int32), ("act_fmt", C.c_int32)]


class LqRopeConfig(C.Structure):
    _fields_ = [("axes", C.c_int32), ("dims", C.c_int32 * 4), ("halves", C.c_int32), ("shared", C.c_int32), ("theta", C.c_double)]


class LqHeads(C.Structure):
    _fields_ = [("in_", C.c_void_p), ("out", C.c_void_p), ("in_seq", C.c_int64), ("in_row", C.c_int64), ("in_head", C.c_int64),
                ("out_seq", C.c_int64), ("out_row", C.c_int64), ("out_head", C.c_int64), ("weight", C.c_void_p), ("bias", C.c_void_p),
                ("heads", C.c_int32)]


class LqQkv(C.Structure):
    _fields_ = [("head_dim", C.c_int32), ("q_heads", C.c_int32), ("kv_heads", C.c_int32), ("sequences", C.c_int32), ("norm", C.c_int32),
                ("eps", C.c_float), ("q_weight", C.c_void_p), ("k_weight", C.c_void_p), ("q_bias", C.c_void_p), ("k_bias", C.c_void_p),
                ("rope", C.c_void_p), ("pos_dev", C.c_void_p)]


class LqKvBatch(C.Structure):
    _fields_ = [("sequences", C.c_int32), ("rows", C.c_int32), ("row_start", C.c_void_p), ("length", C.c_void_p), ("pages", C.c_void_p),
                ("page_stride", C.c_int32)]


class LqKvRows(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_seq", C.c_int64), ("k_row", C.c_int64), ("k_head", C.c_int64),
                ("v_seq", C.c_int64), ("v_row", C.c_int64), ("v_head", C.c_int64)]


class LqAttn(C.Structure):
    _fields_ = [("q", C.c_void_p), ("out", C.c_void_p), ("q_row", C.c_int64), ("q_head", C.c_int64), ("out_row", C.c_int64),
                ("out_head", C.c_int64), ("q_heads", C.c_int32), ("causal", C.c_int32), ("window", C.c_int32), ("sinks", C.c_int32),
                ("scale", C.c_float)]


class LqResidual(C.Structure):
    _fields_ = [("x", C.c_void_p), ("y", C.c_void_p), ("x_out", C.c_void_p), ("h", C.c_void_p), ("x_row", C.c_int64), ("y_row", C.c_int64),
                ("x_out_row", C.c_int64), ("h_row", C.c_int64), ("after_weight", C.c_void_p), ("weight", C.c_void_p), ("bias", C.c_void_p),
                ("gate", C.c_void_p), ("scale", C.c_void_p), ("shift", C.c_void_p), ("mod_seq", C.c_int64), ("rows", C.c_int32),
                ("features", C.c_int32), ("sequences", C.c_int32), ("after", C.c_int32), ("norm", C.c_int32), ("x_dtype", C.c_int32),
                ("y_dtype", C.c_int32), ("h_dtype", C.c_int32), ("mod_dtype", C.c_int32), ("factor", C.c_float), ("eps", C.c_float),
                ("device", C.c_int32)]


# The fields of the structures above in the header's layout: packed at once they take a third of the time that ctypes takes field by field, which
# counts in calls of a few microseconds.
_KV_BATCH, _KV_ROWS, _ATTN = struct.Struct("@iiPPPi4x"), struct.Struct("@PP6q"), struct.Struct("@PP4qiiiif4x")
_RESIDUAL = struct.Struct("@4P4q6Pq9iffi")


class LqError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        detail = f" [{lib().lq_last_cuda_error().decode()}]" if code == 4 else ""
        super().__init__(f"{where}: {lib().lq_status_string(code).decode()} (lq_status {code}){detail}")


_lib = None

_SIGNATURES = {
    "lq_config_default": [C.POINTER(LqConfig), C.c_int32, C.c_int32, C.c_int32, C.c_int32],
    "lq_calibrate": [C.POINTER(LqConfig), C.c_void_p, C.c_void_p, C.POINTER(C.c_void_p), C.c_void_p],
    "lq_layer_import": [C.POINTER(LqConfig), C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                        C.c_void_p, C.c_void_p, C.POINTER(C.c_void_p)],
    "lq_layer_export": [C.c_void_p] * 8,
    "lq_layer_info": [C.c_void_p, C.POINTER(LqConfig)],
    "lq_layer_to_device": [C.c_void_p, C.c_int],
    "lq_layer_free": [C.c_void_p],
    "lq_act_create": [C.c_void_p, C.c_int32, C.c_int, C.POINTER(C.c_void_p)],
    "lq_act_free": [C.c_void_p],
    "lq_quantize_act": [C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p],
    "lq_linear_forward": [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_void_p],
    "lq_linear_forward_host": [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_int, C.c_void_p],
    "lq_linear_forward_host_async": [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_int, C.c_void_p],
    "lq_linear_forward_static": [C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_int, C.c_void_p],
    "lq_adapters_create": [C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_int, C.POINTER(C.c_void_p)],
    "lq_adapters_set": [C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_float, C.c_void_p],
    "lq_adapters_free": [C.c_void_p],
    "lq_rowmap_create": [C.c_int32, C.c_int32, C.c_int, C.POINTER(C.c_void_p)],
    "lq_rowmap_set": [C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p],
    "lq_rowmap_free": [C.c_void_p],
    "lq_adapters_forward": [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_void_p],
    "lq_rope_config_default": [C.POINTER(LqRopeConfig), C.c_int32, C.c_void_p],
    "lq_rope_create": [C.POINTER(LqRopeConfig), C.c_void_p, C.c_void_p, C.c_int, C.POINTER(C.c_void_p)],
    "lq_rope_free": [C.c_void_p],
    "lq_qk_norm_rope": [C.POINTER(LqHeads), C.POINTER(LqHeads), C.c_int32, C.c_int32, C.c_int32, C.c_int, C.c_float, C.c_void_p,
                        C.c_void_p, C.c_int, C.c_int, C.c_void_p],
    "lq_qkv_forward": [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.POINTER(LqQkv), C.c_void_p, C.c_int, C.c_void_p],
    "lq_kvcache_create": [C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_int, C.POINTER(C.c_void_p)],
    "lq_kvcache_free": [C.c_void_p],
    "lq_kvcache_append": [C.c_void_p, C.c_int32, C.POINTER(LqKvBatch), C.POINTER(LqKvRows), C.c_int, C.c_void_p],
    "lq_kvcache_read": [C.c_void_p, C.c_int32, C.POINTER(LqKvBatch), C.c_void_p, C.c_int32, C.POINTER(LqKvRows), C.c_int, C.c_void_p],
    "lq_cache_attention": [C.c_void_p, C.c_int32, C.POINTER(LqKvBatch), C.POINTER(LqAttn), C.c_void_p],
    "lq_residual_norm": [C.POINTER(LqResidual), C.c_void_p],
    "lq_act_export": [C.c_void_p] * 8,
    "lq_get_device_status": [C.c_int, C.POINTER(C.c_int32), C.POINTER(C.c_int32)],
    "lq_set_option": [C.c_char_p, C.c_int32],
    "lq_selftest_wait_timeout": [C.c_int, C.c_void_p],
}
EXPORTED = tuple(_SIGNATURES) + ("lq_status_string", "lq_last_cuda_error", "lq_version")


def lib() -> C.CDLL:
    """The loaded shared library (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} not found: build it with `python -m paper_2604_18117_b200.build`")
        _lib = C.CDLL(LIB_PATH)
        for name, args in _SIGNATURES.items():
            fn = getattr(_lib, name)
            fn.argtypes = args
            fn.restype = C.c_int
        _lib.lq_status_string.argtypes = [C.c_int]
        _lib.lq_status_string.restype = C.c_char_p
        _lib.lq_last_cuda_error.argtypes = []
        _lib.lq_last_cuda_error.restype = C.c_char_p
        _lib.lq_version.argtypes = []
        _lib.lq_version.restype = C.c_int
    return _lib


def _check(code: int, where: str):
    if code != LQ_OK:
        raise LqError(code, where)


def _np_ptr(a):
    return None if a is None else a.ctypes.data_as(C.c_void_p)


def lq_config_default(K: int, N: int, rank: int, branch) -> LqConfig:
    cfg = LqConfig()
    b = BRANCH[branch] if isinstance(branch, str) else int(branch)
    _check(lib().lq_config_default(C.byref(cfg), K, N, rank, b), "lq_config_default")
    return cfg


def lq_calibrate(cfg: LqConfig, W16: np.ndarray, bias16: np.ndarray | None = None, want_trace: bool = False):
    """W16: fp16 [K, N] host array.  Returns (layer handle, trace or None)."""
    W16 = np.ascontiguousarray(W16, dtype=np.float16)
    assert W16.shape == (cfg.K, cfg.N)
    b = None if bias16 is None else np.ascontiguousarray(bias16, dtype=np.float16)
    trace = np.zeros(cfg.steps + 1, dtype=np.float64) if want_trace else None
    h = C.c_void_p()
    _check(lib().lq_calibrate(C.byref(cfg), _np_ptr(W16), _np_ptr(b), C.byref(h), _np_ptr(trace)), "lq_calibrate")
    return h, trace


def pack_nibbles(Wq: np.ndarray) -> np.ndarray:
    """int8 codes [K, N] -> bytes [K, N/2]: column 2j in the low nibble, 2j+1 in the high nibble."""
    u = Wq.astype(np.uint8) & 0xF
    return np.ascontiguousarray(u[:, 0::2] | (u[:, 1::2] << 4))


def unpack_nibbles(P: np.ndarray) -> np.ndarray:
    lo = (P & 0xF).astype(np.int8)
    hi = (P >> 4).astype(np.int8)
    lo = np.where(lo >= 8, lo - 16, lo).astype(np.int8)
    hi = np.where(hi >= 8, hi - 16, hi).astype(np.int8)
    out = np.empty((P.shape[0], P.shape[1] * 2), dtype=np.int8)
    out[:, 0::2], out[:, 1::2] = lo, hi
    return out


# ---- e4m3 / e2m1 byte formats (layout only: the bit patterns of the OCP element formats; no method arithmetic) ----
def _e4m3_table() -> np.ndarray:
    """Value of each of the 256 e4m3 bit patterns (bias 7, subnormals, no infinities; 0x7F / 0xFF are NaN)."""
    t = np.zeros(256, dtype=np.float32)
    for b in range(256):
        e, m = (b >> 3) & 0xF, b & 7
        v = m / 8.0 * 2.0 ** -6 if e == 0 else (1 + m / 8.0) * 2.0 ** (e - 7)
        t[b] = np.nan if (b & 0x7F) == 0x7F else (-v if b & 0x80 else v)
    return t


E4M3_VALUES = _e4m3_table()


def e4m3_decode(codes: np.ndarray) -> np.ndarray:
    """uint8 / int8 e4m3 bit patterns -> float32 values."""
    return E4M3_VALUES[np.asarray(codes).view(np.uint8)]


def e4m3_encode(values: np.ndarray) -> np.ndarray:
    """float values that are exactly representable in e4m3 -> their bit patterns (uint8); raises otherwise."""
    v = np.asarray(values, dtype=np.float32)
    pos = E4M3_VALUES[:0x7F]                                   # ascending non-negative values
    idx = np.searchsorted(pos, np.abs(v))
    idx = np.minimum(idx, 0x7E)
    if not np.array_equal(pos[idx], np.abs(v)):
        raise ValueError("value not representable in e4m3")
    return (idx.astype(np.uint8) | np.where(np.signbit(v), 0x80, 0).astype(np.uint8)).astype(np.uint8)


def pack_e2m1(values: np.ndarray) -> np.ndarray:
    """e2m1 element values [K, N] -> nibbles [K, N/2] (sign, two exponent bits, one mantissa bit), column 2j low."""
    grid = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=np.float32)
    v = np.asarray(values, dtype=np.float32)
    idx = np.searchsorted(grid, np.abs(v))
    idx = np.minimum(idx, 7)
    if not np.array_equal(grid[idx], np.abs(v)):
        raise ValueError("value not representable in e2m1")
    nib = (idx | np.where(np.signbit(v) & (v != 0), 8, 0)).astype(np.uint8)
    return np.ascontiguousarray(nib[:, 0::2] | (nib[:, 1::2] << 4))


def lq_layer_import(cfg: LqConfig, Wq_packed, sw, L1=None, sL1=None, L2=None, sL2=None, bias=None):
    """All arguments are host numpy arrays in the layouts include/lq.h documents."""
    arrs = [np.ascontiguousarray(a) if a is not None else None for a in (Wq_packed, sw, L1, sL1, L2, sL2, bias)]
    h = C.c_void_p()
    _check(lib().lq_layer_import(C.byref(cfg), *[_np_ptr(a) for a in arrs], C.byref(h)), "lq_layer_import")
    return h


def lq_layer_info(layer) -> LqConfig:
    cfg = LqConfig()
    _check(lib().lq_layer_info(layer, C.byref(cfg)), "lq_layer_info")
    return cfg


def lq_layer_export(layer) -> dict:
    cfg = lq_layer_info(layer)
    K, N, r, G = cfg.K, cfg.N, cfg.rank, -(-cfg.K // cfg.group)
    out = {"Wq_packed": np.zeros((K, N // 2), np.uint8), "sw": np.zeros((G, N), np.float16),
           "bias": np.zeros(N, np.float16), "branch": BRANCH_NAME[cfg.branch], "rank": r, "K": K, "N": N}
    L1 = L2 = sL1 = sL2 = None
    if cfg.main_fmt == MAIN_MXFP4 and r > 0:
        L1, L2 = np.zeros((K, r), np.uint8), np.zeros((r, N), np.uint8)               # e4m3 bit patterns
        sL1, sL2 = np.zeros((G, r), np.float32), np.zeros((-(-r // 32), N), np.float32)
    elif cfg.main_fmt == MAIN_MXINT4_A8 and r > 0:
        L1, L2 = np.zeros((K, r), np.int8), np.zeros((r, N), np.int8)                 # integer codes
        sL1, sL2 = np.zeros((G, r), np.float32), np.zeros((-(-r // 32), N), np.float32)   # block scales 2^e
    elif r > 0 and cfg.branch == BRANCH["w16a16"]:
        L1, L2 = np.zeros((K, r), np.float16), np.zeros((r, N), np.float16)
    elif r > 0:
        L1, L2 = np.zeros((K, r), np.int8), np.zeros((r, N), np.int8)
        sL1, sL2 = np.zeros(r, np.float32), np.zeros(N, np.float32)
    _check(lib().lq_layer_export(layer, _np_ptr(out["Wq_packed"]), _np_ptr(out["sw"]), _np_ptr(L1), _np_ptr(sL1),
                                 _np_ptr(L2), _np_ptr(sL2), _np_ptr(out["bias"])), "lq_layer_export")
    out.update(L1=L1, L2=L2, sL1=sL1, sL2=sL2)
    return out


def lq_layer_to_device(layer, device: int = 0):
    _check(lib().lq_layer_to_device(layer, device), "lq_layer_to_device")


def lq_layer_free(layer):
    _check(lib().lq_layer_free(layer), "lq_layer_free")


def lq_act_create(layer, M_max: int, device: int = 0):
    h = C.c_void_p()
    _check(lib().lq_act_create(layer, M_max, device, C.byref(h)), "lq_act_create")
    return h


def lq_act_free(act):
    _check(lib().lq_act_free(act), "lq_act_free")


def lq_quantize_act(layer, X_dev_ptr: int, M: int, act, stream: int = 0):
    _check(lib().lq_quantize_act(layer, C.c_void_p(X_dev_ptr), M, act, C.c_void_p(stream)), "lq_quantize_act")


def lq_linear_forward(layer, act, Y_dev_ptr: int, dtype: int = OUT_F16, stream: int = 0):
    _check(lib().lq_linear_forward(layer, act, C.c_void_p(Y_dev_ptr), dtype, C.c_void_p(stream)), "lq_linear_forward")


def lq_linear_forward_host(layer, act, X_host_ptr: int, M: int, Y_host_ptr: int, dtype: int = OUT_F16, stream: int = 0):
    _check(lib().lq_linear_forward_host(layer, act, C.c_void_p(X_host_ptr), M, C.c_void_p(Y_host_ptr), dtype,
                                        C.c_void_p(stream)), "lq_linear_forward_host")


def lq_linear_forward_host_async(layer, act, X_host_ptr: int, M: int, Y_host_ptr: int, dtype: int = OUT_F16, stream: int = 0):
    _check(lib().lq_linear_forward_host_async(layer, act, C.c_void_p(X_host_ptr), M, C.c_void_p(Y_host_ptr), dtype,
                                        C.c_void_p(stream)), "lq_linear_forward_host_async")


STATIC_SCRATCH_BYTES = 8 << 20


def lq_linear_forward_static(layer, X_dev_ptr: int, M: int, Y_dev_ptr: int, dtype: int = OUT_F16, stream: int = 0):
    """Whole forward without any allocation at call time: the activation record lives in a fixed
    device array inside the library (for callers whose memory pool forbids raw allocations).
    Raises LqError(code 2) when M x K does not fit the array; calls must not overlap on the GPU."""
    _check(lib().lq_linear_forward_static(layer, C.c_void_p(X_dev_ptr), M, C.c_void_p(Y_dev_ptr), dtype,
                                          C.c_void_p(stream)), "lq_linear_forward_static")


def lq_adapters_create(K: int, N: int, max_rank: int, slots: int, device: int = 0):
    h = C.c_void_p()
    _check(lib().lq_adapters_create(K, N, max_rank, slots, device, C.byref(h)), "lq_adapters_create")
    return h


def lq_adapters_set(adapters, slot: int, rank: int, A_dev_ptr: int | None, B_dev_ptr: int | None, scale: float = 1.0, stream: int = 0):
    """A fp16 [K, rank] and B fp16 [rank, N] on the device; rank 0 empties the slot."""
    _check(lib().lq_adapters_set(adapters, slot, rank, C.c_void_p(A_dev_ptr), C.c_void_p(B_dev_ptr), scale, C.c_void_p(stream)),
           "lq_adapters_set")


def lq_adapters_free(adapters):
    _check(lib().lq_adapters_free(adapters), "lq_adapters_free")


def lq_rowmap_create(M_max: int, slots: int, device: int = 0):
    h = C.c_void_p()
    _check(lib().lq_rowmap_create(M_max, slots, device, C.byref(h)), "lq_rowmap_create")
    return h


def lq_rowmap_set(rowmap, row_adapter_dev_ptr: int, M: int, stream: int = 0):
    _check(lib().lq_rowmap_set(rowmap, row_adapter_dev_ptr, M, stream), "lq_rowmap_set")


def lq_rowmap_free(rowmap):
    _check(lib().lq_rowmap_free(rowmap), "lq_rowmap_free")


def lq_adapters_forward(adapters, rowmap, X_dev_ptr: int, Y0_dev_ptr: int, Y_dev_ptr: int, dtype: int = OUT_F16, stream: int = 0):
    """Y = Y0 + each row's adapter on X; Y may be Y0 itself."""
    _check(lib().lq_adapters_forward(adapters, rowmap, X_dev_ptr, Y0_dev_ptr, Y_dev_ptr, dtype, stream), "lq_adapters_forward")


def lq_rope_config_default(dims, theta: float = 10000.0, halves: bool = False, shared: bool = False) -> LqRopeConfig:
    cfg = LqRopeConfig()
    d = np.ascontiguousarray(dims, dtype=np.int32)
    _check(lib().lq_rope_config_default(C.byref(cfg), d.size, _np_ptr(d)), "lq_rope_config_default")
    cfg.theta, cfg.halves, cfg.shared = theta, int(halves), int(shared)
    return cfg


def lq_rope_create(cfg: LqRopeConfig, device: int = 0, freq: np.ndarray | None = None, axis: np.ndarray | None = None):
    """freq, axis: host arrays with an entry for each rotated pair, in place of the configuration's."""
    pairs = sum(cfg.dims[: max(0, min(cfg.axes, 4))]) // 2
    f = None if freq is None else np.ascontiguousarray(freq, dtype=np.float64)
    a = None if axis is None else np.ascontiguousarray(axis, dtype=np.int32)
    assert all(v is None or v.shape == (pairs,) for v in (f, a))
    h = C.c_void_p()
    _check(lib().lq_rope_create(C.byref(cfg), _np_ptr(f), _np_ptr(a), device, C.byref(h)), "lq_rope_create")
    return h


def lq_rope_free(rope):
    _check(lib().lq_rope_free(rope), "lq_rope_free")


def lq_heads(in_ptr: int, in_strides, out_ptr: int, out_strides, heads: int, weight_ptr: int | None = None,
             bias_ptr: int | None = None) -> LqHeads:
    """The queries or keys of a call; strides of sequence, row and head in elements."""
    return LqHeads(in_ptr, out_ptr, *in_strides, *out_strides, weight_ptr, bias_ptr, heads)


def lq_qk_norm_rope(q: LqHeads | None, k: LqHeads | None, head_dim: int, sequences: int, seq_len: int, norm: int, eps: float, rope,
                    pos_dev_ptr: int | None, in_dtype: int = OUT_F16, out_dtype: int = OUT_F16, stream: int = 0):
    _check(lib().lq_qk_norm_rope(q, k, head_dim, sequences, seq_len, norm, eps, rope, pos_dev_ptr, in_dtype, out_dtype, stream), "lq_qk_norm_rope")


def lq_qkv(head_dim: int, q_heads: int, kv_heads: int, sequences: int, norm: int, eps: float, rope, pos_dev_ptr: int | None = None,
           q_weight_ptr: int | None = None, k_weight_ptr: int | None = None, q_bias_ptr: int | None = None, k_bias_ptr: int | None = None) -> LqQkv:
    return LqQkv(head_dim, q_heads, kv_heads, sequences, norm, eps, q_weight_ptr, k_weight_ptr, q_bias_ptr, k_bias_ptr, rope, pos_dev_ptr)


def lq_qkv_forward(layer, act, X_dev_ptr: int, M: int, adapters, rowmap, qkv: LqQkv, Y_dev_ptr: int, dtype: int = OUT_F16, stream: int = 0):
    """Quantizer, GEMM, the rows' adapters (both handles, or None), norm and rotation of queries and keys: Y [M, N]."""
    _check(lib().lq_qkv_forward(layer, act, X_dev_ptr, M, adapters, rowmap, qkv, Y_dev_ptr, dtype, stream), "lq_qkv_forward")


def lq_kvcache_create(layers: int, pages: int, page_tokens: int, kv_heads: int, head_dim: int, device: int = 0):
    h = C.c_void_p()
    _check(lib().lq_kvcache_create(layers, pages, page_tokens, kv_heads, head_dim, device, C.byref(h)), "lq_kvcache_create")
    return h


def lq_kvcache_free(cache):
    _check(lib().lq_kvcache_free(cache), "lq_kvcache_free")


def lq_kvbatch(sequences: int, rows: int, length_ptr: int, pages_ptr: int, page_stride: int, row_start_ptr: int | None = None) -> LqKvBatch:
    """The sequences of a step: int32 arrays on the device; without row_start every sequence has rows / sequences rows."""
    return LqKvBatch.from_buffer_copy(_KV_BATCH.pack(sequences, rows, row_start_ptr or 0, length_ptr, pages_ptr, page_stride))


def lq_kvrows(k_ptr: int | None, k_strides, v_ptr: int | None, v_strides) -> LqKvRows:
    """Keys and values; strides of sequence (outputs alone), row and head in elements."""
    return LqKvRows.from_buffer_copy(_KV_ROWS.pack(k_ptr or 0, v_ptr or 0, *k_strides, *v_strides))


def lq_kvcache_append(cache, layer: int, batch: LqKvBatch, rows: LqKvRows, dtype: int = OUT_F16, stream: int = 0):
    """Quantises the batch's rows into the cache as each sequence's last tokens."""
    _check(lib().lq_kvcache_append(cache, layer, batch, rows, dtype, stream), "lq_kvcache_append")


def lq_kvcache_read(cache, layer: int, batch: LqKvBatch, begin_dev_ptr: int | None, max_tokens: int, rows: LqKvRows, dtype: int = OUT_F16, stream: int = 0):
    """Tokens from begin (None: the first) to each sequence's length, at most max_tokens, as values."""
    _check(lib().lq_kvcache_read(cache, layer, batch, begin_dev_ptr, max_tokens, rows, dtype, stream), "lq_kvcache_read")


def lq_attn(q_ptr: int, q_strides, out_ptr: int, out_strides, q_heads: int, scale: float, causal: bool = True, window: int = 0, sinks: int = 0) -> LqAttn:
    """Queries and output of an attention call; strides of row and head in elements."""
    return LqAttn.from_buffer_copy(_ATTN.pack(q_ptr, out_ptr, *q_strides, *out_strides, q_heads, causal, window, sinks, scale))


def lq_cache_attention(cache, layer: int, batch: LqKvBatch, attn: LqAttn, stream: int = 0):
    _check(lib().lq_cache_attention(cache, layer, batch, attn, stream), "lq_cache_attention")


def lq_residual(rows: int, features: int, x_ptr: int, x_out_ptr: int | None, h_ptr: int | None, y_ptr: int | None = None, sequences: int = 1,
                after: int = NORM_NONE, after_weight_ptr: int | None = None, factor: float = 1.0, gate_ptr: int | None = None,
                norm: int = NORM_NONE, weight_ptr: int | None = None, bias_ptr: int | None = None, scale_ptr: int | None = None,
                shift_ptr: int | None = None, mod_seq: int = 0, eps: float = 1e-6, x_dtype: int = OUT_F16, y_dtype: int = OUT_F16,
                h_dtype: int = OUT_F16, mod_dtype: int = OUT_F16, strides=None, device: int = 0) -> LqResidual:
    """strides: of the rows of x, y, x_out and h in elements (None: rows follow each other)."""
    x_row, y_row, x_out_row, h_row = strides or (features, features, features, features)
    return LqResidual.from_buffer_copy(_RESIDUAL.pack(
        x_ptr, y_ptr or 0, x_out_ptr or 0, h_ptr or 0, x_row, y_row, x_out_row, h_row, after_weight_ptr or 0, weight_ptr or 0, bias_ptr or 0, gate_ptr or 0,
        scale_ptr or 0, shift_ptr or 0, mod_seq, rows, features, sequences, after, norm, x_dtype, y_dtype, h_dtype, mod_dtype, factor, eps, device))


def lq_residual_norm(residual: LqResidual, stream: int = 0):
    """x' = x + factor * gate * N1(y) and h = (N2(x') * weight + bias) * (1 + scale) + shift."""
    _check(lib().lq_residual_norm(residual, stream), "lq_residual_norm")


def lq_act_export(act, M: int, cfg: LqConfig, stream: int = 0) -> dict:
    K, r, G = cfg.K, cfg.rank, -(-cfg.K // cfg.group)
    if cfg.main_fmt in (MAIN_MXFP4, MAIN_MXINT4_A8):
        # MXFP: qx / tq are e4m3 bit patterns (decode with e4m3_decode); integer MX with 8-bit activations: the int8 codes.
        # sx: the int16 block exponents of X; sT: the block exponents of the rank-r intermediate as floats [M, ceil(r/32)]
        out = {"qx": np.zeros((M, K), np.int8), "sx": np.zeros((M, G), np.int16), "qb": None, "sXb": None, "tq": None, "sT": None}
        if r > 0 and cfg.branch != BRANCH["none"]:
            out["tq"] = np.zeros((M, r), np.int8)
            out["sT"] = np.zeros((M, -(-r // 32)), np.float32)
        _check(lib().lq_act_export(act, _np_ptr(out["qx"]), _np_ptr(out["sx"]), None, None, _np_ptr(out["tq"]),
                                   _np_ptr(out["sT"]), C.c_void_p(stream)), "lq_act_export")
        return out
    # SINT4: fp16 group scales; MXINT4 (group 32): int16 block exponents e (scale 2^e)
    out = {"qx": np.zeros((M, K), np.int8), "sx": np.zeros((M, G), np.int16 if cfg.group == 32 else np.float16)}
    qb = sXb = tq = sT = None
    if r > 0 and cfg.branch != BRANCH["none"]:
        f16 = cfg.branch == BRANCH["w16a16"]
        tq = np.zeros((M, r), np.float16 if f16 else np.int8)
        sT = np.zeros(M, np.float32)
        if not f16:
            qb, sXb = np.zeros((M, K), np.int8), np.zeros(M, np.float32)
    _check(lib().lq_act_export(act, _np_ptr(out["qx"]), _np_ptr(out["sx"]), _np_ptr(qb), _np_ptr(sXb), _np_ptr(tq),
                               _np_ptr(sT), C.c_void_p(stream)), "lq_act_export")
    out.update(qb=qb, sXb=sXb, tq=tq, sT=sT)
    return out


def lq_get_device_status(device: int = 0):
    code, stage = C.c_int32(), C.c_int32()
    _check(lib().lq_get_device_status(device, C.byref(code), C.byref(stage)), "lq_get_device_status")
    return code.value, stage.value


def lq_selftest_wait_timeout(device: int = 0, stream: int = 0):
    _check(lib().lq_selftest_wait_timeout(device, C.c_void_p(stream)), "lq_selftest_wait_timeout")


def lq_set_option(name: str, value: int):
    _check(lib().lq_set_option(name.encode(), value), "lq_set_option")


def lq_version() -> int:
    return lib().lq_version()
