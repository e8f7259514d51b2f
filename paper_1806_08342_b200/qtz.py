"""ctypes binding of libqtz (the C ABI in ``include/qtz.h``).

Argument marshalling only: every function takes torch CUDA tensors (PyTorch is used
for device memory and streams), passes their pointers and sizes to the entry point of
the same name, and raises :class:`QtzError` on a non-zero status.  There is no
fallback: if ``libqtz.so`` has not been built this module raises on first use.
"""
from __future__ import annotations

import ctypes
import os
import weakref
from ctypes import POINTER, Structure, byref, c_char_p, c_double, c_float, c_int32, c_int64, c_void_p

import numpy as np
import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libqtz.so")

U8, S8, S4_PACKED, S32, U4_PACKED, U16, S16 = 0, 1, 2, 3, 4, 5, 6
W_S8_PER_CHANNEL_SYM, W_U8_PER_LAYER_ASYM, W_S4_PACKED_PER_CHANNEL_SYM = 0, 1, 2
OUT_U8, OUT_S32_RAW = 0, 1
ACT_NONE, ACT_RELU, ACT_RELU6 = 0, 1, 2
F32, F16, BF16 = 16, 17, 18
DEVICE_TIMEOUT = -7
FTYPES = {torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16}
E4M3 = torch.float8_e4m3fn

QPARAMS = np.dtype([("scale", "<f4"), ("zero_point", "<i4"), ("min_nudged", "<f4"), ("max_nudged", "<f4")])


class ConvDesc(Structure):
    _fields_ = [(n, c_int32) for n in ("batch", "h", "w", "c", "c_pitch_in", "n", "c_pitch_out", "kh", "kw",
                                       "stride", "pad", "wkind", "outkind")]


class Residual(Structure):
    _fields_ = [(n, c_int32) for n in ("t_zero_point", "t_act_min", "t_act_max", "t_mult", "s_zero_point", "s_mult", "rshift")]


class LinearDesc(Structure):
    _fields_ = [(n, c_int32) for n in ("n", "k", "group", "wdtype", "ftype")]


class KvCacheDesc(Structure):
    _fields_ = [(n, c_void_p) for n in ("k_dev", "v_dev", "k_scale_dev", "v_scale_dev")] + \
               [(n, c_int32) for n in ("blocks", "kv_heads", "block_tokens", "head_dim")]


class QtzError(RuntimeError):
    def __init__(self, code, what, detail=""):
        super().__init__(f"{what}: status {code} ({detail})")
        self.code = code


_lib = None

# name -> (restype, argtypes); every symbol declared in include/qtz.h
SIGNATURES = {
    "qtz_create": (c_int32, [POINTER(c_void_p), ctypes.c_int]),
    "qtz_destroy": (c_int32, [c_void_p]),
    "qtz_status_string": (c_char_p, [c_int32]),
    "qtz_last_error": (c_char_p, [c_void_p]),
    "qtz_last_device_status": (c_int32, [c_void_p, POINTER(c_int32), c_void_p]),
    "qtz_set_wait_budget": (c_int32, [c_void_p, c_int64]),
    "qtz_selftest_wait_timeout": (c_int32, [c_void_p, c_int64, c_void_p]),
    "qtz_probe_int8_peak": (c_int32, [c_void_p, c_int32, c_int32, POINTER(c_double), POINTER(c_float), c_void_p]),
    "qtz_probe_requant_rate": (c_int32, [c_void_p, c_int32, POINTER(c_double), POINTER(c_double), c_void_p]),
    "qtz_calibrate_minmax": (c_int32, [c_void_p, c_void_p, c_int64, c_int64, c_int64, c_int32, c_int32, c_void_p,
                                       c_void_p]),
    "qtz_minmax": (c_int32, [c_void_p, c_void_p, c_int64, c_int64, c_int64, c_void_p, c_void_p, c_void_p]),
    "qtz_minmax_static": (c_int32, [c_void_p, c_int64, c_void_p, c_void_p]),
    "qtz_minmax_static_max_count": (c_int64, []),
    "qtz_range_state_bytes": (c_int64, [c_int64]),
    "qtz_range_reset": (c_int32, [c_void_p, c_void_p, c_int64, c_void_p]),
    "qtz_range_accumulate": (c_int32, [c_void_p, c_void_p, c_int64, c_int64, c_int64, c_double, c_void_p, c_void_p]),
    "qtz_range_finish": (c_int32, [c_void_p, c_void_p, c_int64, c_int32, c_int32, c_void_p, c_void_p, c_void_p,
                                   POINTER(c_int32), c_void_p]),
    "qtz_params_from_range": (c_int32, [c_float, c_float, c_int32, c_int32, c_void_p]),
    "qtz_quantize_tensor": (c_int32, [c_void_p, c_void_p, c_int64, c_int64, c_int64, c_void_p, c_int32, c_int32,
                                      c_void_p, c_void_p]),
    "qtz_dequantize": (c_int32, [c_void_p, c_void_p, c_int32, c_int64, c_int64, c_int64, c_void_p, c_void_p,
                                 c_void_p]),
    "qtz_fold_batchnorm": (c_int32, [c_void_p] * 7 + [c_float, c_int64, c_int64, c_void_p, c_void_p, c_void_p]),
    "qtz_quantize_bias": (c_int32, [c_void_p, c_void_p, c_int64, c_float, c_void_p, c_int32, c_void_p, c_void_p]),
    "qtz_quantize_multiplier": (c_int32, [c_double, POINTER(c_int32), POINTER(c_int32)]),
    "qtz_activation_range": (c_int32, [c_int32, c_float, c_int32, POINTER(c_int32), POINTER(c_int32)]),
    "qtz_activation_range_bits": (c_int32, [c_int32, c_float, c_int32, c_int32, POINTER(c_int32), POINTER(c_int32)]),
    "qtz_pack_u4": (c_int32, [c_void_p, c_void_p, c_int64, c_int32, c_int32, c_void_p, c_int32, c_void_p]),
    "qtz_unpack_u4": (c_int32, [c_void_p, c_void_p, c_int64, c_int32, c_int32, c_void_p, c_int32, c_void_p]),
    "qtz_add_params": (c_int32, [c_float, c_float, c_float, POINTER(c_int32), POINTER(c_int32), POINTER(c_int32)]),
    "qtz_range_after_activation": (c_int32, [c_float, c_float, c_int32, POINTER(c_float), POINTER(c_float)]),
    "qtz_add_output_range": (c_int32, [c_void_p, c_void_p, c_int32, POINTER(c_float), POINTER(c_float)]),
    "qtz_accumulator_scales": (c_int32, [c_float, c_void_p, c_int64, c_void_p]),
    "qtz_requant_multipliers": (c_int32, [c_float, c_void_p, c_int64, c_float, c_void_p, c_void_p]),
    "qtz_avgpool_multiplier": (c_int32, [c_int32, c_float, c_float, POINTER(c_int32), POINTER(c_int32)]),
    "qtz_conv_create": (c_int32, [c_void_p, POINTER(ConvDesc), c_int32, c_void_p, c_void_p, c_void_p, c_void_p,
                                  c_void_p, POINTER(c_void_p), c_void_p]),
    "qtz_conv_destroy": (c_int32, [c_void_p]),
    "qtz_conv_plan_kernel": (c_char_p, [c_void_p]),
    "qtz_conv_plan_detail": (c_char_p, [c_void_p]),
    "qtz_conv_set_profile_events": (c_int32, [c_void_p, c_void_p, c_void_p]),
    "qtz_conv2d_u8": (c_int32, [c_void_p, c_void_p, c_int32, c_void_p, c_int32, c_int32, c_int32, c_void_p]),
    "qtz_conv2d_add_u8": (c_int32, [c_void_p, c_void_p, c_int32, POINTER(Residual), c_void_p, c_void_p, c_int32, c_int32, c_int32,
                                    c_void_p]),
    "qtz_depthwise_u8": (c_int32, [c_void_p, c_void_p, c_int32, c_void_p, c_int32, c_int32, c_int32, c_void_p]),
    "qtz_conv2d_dw_pw_u8": (c_int32, [c_void_p, c_void_p, c_void_p, c_int32, c_int32, c_int32, c_int32, c_void_p, c_int32, c_int32,
                                      c_int32, c_void_p]),
    "qtz_add_u8": (c_int32, [c_void_p, c_void_p, c_int32, c_int32, c_void_p, c_int32, c_int32, c_int32, c_void_p,
                             c_int32, c_int32, c_int32, c_int64, c_int32, c_int32, c_void_p]),
    "qtz_simquant": (c_int32, [c_void_p, c_void_p, c_int64, c_int64, c_int64, c_void_p, c_int32, c_int32, c_void_p, c_void_p]),
    "qtz_sqnr": (c_int32, [c_void_p, c_void_p, c_void_p, c_int64, c_int64, c_int64, c_void_p, c_void_p]),
    "qtz_ema_update": (c_int32, [c_void_p, c_void_p, c_void_p, c_void_p, c_int64, c_double, POINTER(c_int32)]),
    "qtz_rescale_u8": (c_int32, [c_void_p, c_void_p, c_int32, c_int32, c_int32, c_void_p, c_int32, c_int32, c_int32, c_int64,
                                 c_int32, c_int32, c_int32, c_void_p]),
    "qtz_maxpool_u8": (c_int32, [c_void_p, c_void_p, c_void_p] + [c_int32] * 8 + [c_void_p]),
    "qtz_global_avgpool_u8": (c_int32, [c_void_p, c_void_p, c_int32, c_void_p] + [c_int32] * 7 + [c_void_p]),
    "qtz_linear_create": (c_int32, [c_void_p, POINTER(LinearDesc), c_void_p, c_void_p, c_void_p, c_void_p, POINTER(c_void_p), c_void_p]),
    "qtz_linear_destroy": (c_int32, [c_void_p]),
    "qtz_linear_w4": (c_int32, [c_void_p, c_void_p, c_int64, c_int64, c_void_p, c_int64, c_void_p]),
    "qtz_f8_rmsnorm": (c_int32, [c_void_p, c_void_p, c_int64, c_void_p, c_int64, c_void_p, c_float, c_int64, c_int32, c_int32, c_void_p, c_int64,
                                 c_void_p, c_int64, c_void_p, c_int64, c_void_p, c_int64, c_void_p]),
    "qtz_f8_quantize": (c_int32, [c_void_p, c_void_p, c_int64, c_void_p, c_int64, c_int64, c_int32, c_int32, c_void_p, c_int64, c_void_p, c_int64,
                                  c_void_p]),
    "qtz_f8_quantize_weights": (c_int32, [c_void_p, c_void_p, c_int64, c_int32, c_int32, c_int32, c_void_p, c_void_p, c_void_p]),
    "qtz_f8_linear_create": (c_int32, [c_void_p, c_int32, c_int32, c_void_p, c_int64, c_void_p, c_void_p, c_int32, POINTER(c_void_p), c_void_p]),
    "qtz_f8_linear_destroy": (c_int32, [c_void_p]),
    "qtz_f8_linear": (c_int32, [c_void_p, c_void_p, c_int64, c_void_p, c_int64, c_int64, c_int64, c_void_p, c_int64, c_int32, c_void_p]),
    "qtz_kv_schedule": (c_int32, [c_void_p, c_void_p, c_void_p, c_int32, c_int32, c_void_p, c_int32, c_void_p, c_void_p, c_void_p,
                                  c_void_p, c_void_p, c_int64, c_void_p, c_void_p]),
    "qtz_kv_append": (c_int32, [c_void_p, POINTER(KvCacheDesc), c_void_p, c_int64, c_int64, c_void_p, c_int64, c_int64, c_int32, c_void_p,
                                c_int64, c_void_p]),
    "qtz_kv_read": (c_int32, [c_void_p, POINTER(KvCacheDesc), c_void_p, c_int64, c_int32, c_void_p, c_void_p, c_void_p]),
    "qtz_kv_attention_workspace_bytes": (c_int64, [c_void_p, POINTER(KvCacheDesc)]),
    "qtz_kv_attention": (c_int32, [c_void_p, POINTER(KvCacheDesc), c_void_p, c_int64, c_int64, c_int32, c_int32, c_void_p, c_void_p, c_int32,
                                   c_int64, c_void_p, c_int32, c_float, c_int32, c_void_p, c_int64, c_int64, c_void_p, c_void_p, c_void_p]),
}


def load_library():
    """Opens libqtz.so and types its symbols.  Raises if the library has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_1806_08342_b200.build` "
                               "(there is no CPU fallback)")
        lib = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = res, args
        _lib = lib
    return _lib


def _stream():
    return c_void_p(torch.cuda.current_stream().cuda_stream)


def _ptr(t):
    return None if t is None else c_void_p(t.data_ptr())


def _np(a):
    return None if a is None else a.ctypes.data_as(c_void_p)


def _view(shape, axis):
    if axis is None:
        return 1, 1, int(np.prod(shape, dtype=np.int64))
    axis %= len(shape)
    return (int(np.prod(shape[:axis], dtype=np.int64)), int(shape[axis]),
            int(np.prod(shape[axis + 1:], dtype=np.int64)))


def _check_dev(*ts):
    for t in ts:
        if t is not None and (not t.is_cuda or not t.is_contiguous()):
            raise ValueError("expected contiguous CUDA tensors")


# The serving calls are short on the GPU: their checks stay cheap (get_device is -1 for a tensor that is not on a GPU).
def _check_on(device, dtype, *ts):
    for t in ts:
        if t.dtype is not dtype or t.get_device() != device:
            raise ValueError(f"expected {dtype} tensors on cuda:{device}, got {t.dtype} on {t.device}")


def _check_flat(device, dtype, *ts):
    for t in ts:
        if t.dtype is not dtype or t.get_device() != device or not t.is_contiguous():
            raise ValueError(f"expected contiguous {dtype} tensors on cuda:{device}, got {t.dtype} on {t.device}")


def _raw_stream(device):
    return torch._C._cuda_getCurrentRawStream(device)


# ---- host-only helpers ------------------------------------------------------------------
def quantize_multiplier(real_multiplier):
    m, r = c_int32(), c_int32()
    rc = load_library().qtz_quantize_multiplier(float(real_multiplier), byref(m), byref(r))
    if rc:
        raise QtzError(rc, "qtz_quantize_multiplier")
    return m.value, r.value


def activation_range(kind, y_scale, y_zero_point):
    lo, hi = c_int32(), c_int32()
    rc = load_library().qtz_activation_range(kind, float(y_scale), int(y_zero_point), byref(lo), byref(hi))
    if rc:
        raise QtzError(rc, "qtz_activation_range")
    return lo.value, hi.value


def activation_range_bits(kind, y_scale, y_zero_point, bits):
    lo, hi = c_int32(), c_int32()
    rc = load_library().qtz_activation_range_bits(kind, float(y_scale), int(y_zero_point), int(bits), byref(lo), byref(hi))
    if rc:
        raise QtzError(rc, "qtz_activation_range_bits")
    return lo.value, hi.value


def add_params(a_scale, b_scale, y_scale):
    ma, mb, r = c_int32(), c_int32(), c_int32()
    rc = load_library().qtz_add_params(float(a_scale), float(b_scale), float(y_scale), byref(ma), byref(mb), byref(r))
    if rc:
        raise QtzError(rc, "qtz_add_params")
    return ma.value, mb.value, r.value


def range_after_activation(lo, hi, kind):
    a, b = c_float(), c_float()
    rc = load_library().qtz_range_after_activation(float(lo), float(hi), int(kind), byref(a), byref(b))
    if rc:
        raise QtzError(rc, "qtz_range_after_activation")
    return a.value, b.value


def add_output_range(a_params, b_params, kind):
    pa = np.ascontiguousarray(np.atleast_1d(a_params), dtype=QPARAMS)
    pb = np.ascontiguousarray(np.atleast_1d(b_params), dtype=QPARAMS)
    lo, hi = c_float(), c_float()
    rc = load_library().qtz_add_output_range(_np(pa), _np(pb), int(kind), byref(lo), byref(hi))
    if rc:
        raise QtzError(rc, "qtz_add_output_range")
    return lo.value, hi.value


def accumulator_scales(x_scale, w_params):
    wp = np.ascontiguousarray(np.atleast_1d(w_params), dtype=QPARAMS)
    out = np.zeros(wp.shape[0], QPARAMS)
    rc = load_library().qtz_accumulator_scales(float(x_scale), _np(wp), wp.shape[0], _np(out))
    if rc:
        raise QtzError(rc, "qtz_accumulator_scales")
    return out


def requant_multipliers(x_scale, w_params, y_scale):
    wp = np.ascontiguousarray(np.atleast_1d(w_params), dtype=QPARAMS)
    mult, rshift = np.zeros(wp.shape[0], np.int32), np.zeros(wp.shape[0], np.int32)
    rc = load_library().qtz_requant_multipliers(float(x_scale), _np(wp), wp.shape[0], float(y_scale), _np(mult), _np(rshift))
    if rc:
        raise QtzError(rc, "qtz_requant_multipliers")
    return mult, rshift


def avgpool_multiplier(hw, x_scale, y_scale):
    m, r = c_int32(), c_int32()
    rc = load_library().qtz_avgpool_multiplier(int(hw), float(x_scale), float(y_scale), byref(m), byref(r))
    if rc:
        raise QtzError(rc, "qtz_avgpool_multiplier")
    return m.value, r.value


def ema_update(state_lo, state_hi, batch_lo, batch_hi, decay, initialised):
    """Moving average of per-batch ranges (Section 2.5): updates the fp64 state arrays in place and
    returns the new `initialised` flag."""
    assert state_lo.dtype == np.float64 and state_hi.dtype == np.float64 and state_lo.shape == state_hi.shape
    batch_lo = np.ascontiguousarray(batch_lo, dtype=np.float32)
    batch_hi = np.ascontiguousarray(batch_hi, dtype=np.float32)
    assert batch_lo.size == state_lo.size and batch_hi.size == state_lo.size
    flag = c_int32(int(bool(initialised)))
    rc = load_library().qtz_ema_update(_np(state_lo), _np(state_hi), _np(batch_lo), _np(batch_hi), state_lo.size,
                                       float(decay), ctypes.byref(flag))
    if rc != 0:
        raise QtzError(rc, "qtz_ema_update")
    return bool(flag.value)


def params_from_range(lo, hi, bits=8, symmetric=False):
    q = np.zeros(1, QPARAMS)
    rc = load_library().qtz_params_from_range(float(lo), float(hi), bits, int(symmetric), _np(q))
    if rc:
        raise QtzError(rc, "qtz_params_from_range")
    return q[0]


def minmax_static(x, out=None):
    """qtz_minmax_static on the current device and stream.  `x`: fp32 CUDA tensor; returns a 3-word
    CUDA tensor (lo, hi, non-finite flag bits viewed as float).  Allocates only if `out` is None --
    pass a preallocated 3-element fp32 tensor to keep the call allocation-free."""
    _check_dev(x, out)
    assert x.dtype == torch.float32
    if out is None:
        out = torch.empty(3, dtype=torch.float32, device=x.device)
    rc = load_library().qtz_minmax_static(_ptr(x), x.numel(), _ptr(out), _stream())
    if rc:
        raise QtzError(rc, "qtz_minmax_static", load_library().qtz_status_string(rc).decode())
    return out


class Handle:
    """Owns a qtz_handle on one CUDA device."""

    def __init__(self, device: int = 0):
        self.lib = load_library()
        self.h = c_void_p()
        self.device = device
        self._caches = weakref.WeakSet()
        rc = self.lib.qtz_create(byref(self.h), device)
        if rc:
            raise QtzError(rc, "qtz_create", self.lib.qtz_status_string(rc).decode())

    def close(self):
        if self.h:
            self.lib.qtz_destroy(self.h)
            self.h = c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _chk(self, rc, what):
        if rc:
            detail = self.lib.qtz_status_string(rc).decode()
            if rc == -6:
                detail += ": " + self.lib.qtz_last_error(self.h).decode()
            raise QtzError(rc, what, detail)

    def device_status(self):
        """(status, site) of what device code has recorded, (0, 0) for nothing.  After a timeout the workspaces of this handle's
        caches are made ready for the next call."""
        site = c_int32()
        rc = self.lib.qtz_last_device_status(self.h, byref(site), _stream())
        if rc == DEVICE_TIMEOUT:
            for cache in list(self._caches):
                cache.reset_workspace()
        return rc, site.value

    def set_wait_budget(self, cycles):
        self._chk(self.lib.qtz_set_wait_budget(self.h, int(cycles)), "qtz_set_wait_budget")

    def selftest_wait_timeout(self, budget_cycles):
        self._chk(self.lib.qtz_selftest_wait_timeout(self.h, int(budget_cycles), _stream()), "qtz_selftest_wait_timeout")

    def probe_int8_peak(self, mmas_per_cta=32768, launches=10):
        """(TOP/s, ms) of tcgen05.mma kind::i8 issued back to back on shared-memory resident operands."""
        tops, ms = c_double(), c_float()
        self._chk(self.lib.qtz_probe_int8_peak(self.h, int(mmas_per_cta), int(launches), byref(tops), byref(ms), _stream()),
                  "qtz_probe_int8_peak")
        return tops.value, ms.value

    def probe_requant_rate(self, kind):
        """(outputs per clock and SM at the maximum clock, outputs per second) of the requantising arithmetic."""
        a, b = c_double(), c_double()
        self._chk(self.lib.qtz_probe_requant_rate(self.h, int(kind), byref(a), byref(b), _stream()), "qtz_probe_requant_rate")
        return a.value, b.value

    def calibrate_minmax(self, x, axis=None, bits=8, symmetric=False):
        _check_dev(x)
        assert x.dtype == torch.float32
        o, a, i = _view(x.shape, axis)
        out = np.zeros(a, QPARAMS)
        self._chk(self.lib.qtz_calibrate_minmax(self.h, _ptr(x), o, a, i, bits, int(symmetric), _np(out),
                                                _stream()), "qtz_calibrate_minmax")
        return out

    def minmax(self, x, axis=None):
        _check_dev(x)
        assert x.dtype == torch.float32
        o, a, i = _view(x.shape, axis)
        lo, hi = np.zeros(a, np.float32), np.zeros(a, np.float32)
        self._chk(self.lib.qtz_minmax(self.h, _ptr(x), o, a, i, _np(lo), _np(hi), _stream()), "qtz_minmax")
        return lo, hi

    def range_state(self, axis_len=1):
        """A zeroed device buffer for range_accumulate (torch owns the memory)."""
        n = self.lib.qtz_range_state_bytes(int(axis_len))
        return torch.zeros(n // 8, dtype=torch.float64, device=f"cuda:{self.device}")

    def range_reset(self, state, axis_len=1):
        self._chk(self.lib.qtz_range_reset(self.h, _ptr(state), int(axis_len), _stream()), "qtz_range_reset")

    def range_accumulate(self, x, state, decay, axis=None):
        """Folds the min/max of batch `x` into the device-resident moving average; does not wait."""
        _check_dev(x, state)
        assert x.dtype == torch.float32
        o, a, i = _view(x.shape, axis)
        self._chk(self.lib.qtz_range_accumulate(self.h, _ptr(x), o, a, i, float(decay), _ptr(state), _stream()),
                  "qtz_range_accumulate")

    def range_finish(self, state, axis_len=1, bits=8, symmetric=False):
        """One blocking read: (lo, hi, params, batches) of the averaged ranges."""
        lo, hi = np.zeros(axis_len, np.float32), np.zeros(axis_len, np.float32)
        params = np.zeros(axis_len, QPARAMS)
        batches = c_int32()
        self._chk(self.lib.qtz_range_finish(self.h, _ptr(state), int(axis_len), bits, int(symmetric), _np(lo), _np(hi),
                                            _np(params), byref(batches), _stream()), "qtz_range_finish")
        return lo, hi, params, batches.value

    def quantize_tensor(self, x, params, axis=None, out_dtype=U8, restrict_range=False, out=None):
        _check_dev(x, out)
        assert x.dtype == torch.float32
        params = np.ascontiguousarray(np.atleast_1d(params), dtype=QPARAMS)
        o, a, i = _view(x.shape, axis)
        assert params.shape[0] == a
        if out is None:
            if out_dtype in (S4_PACKED, U4_PACKED):
                run = i if i > 1 else a
                out = torch.empty((x.numel() // run) * ((run + 1) // 2), dtype=torch.uint8, device=x.device)
            else:
                out = torch.empty(x.shape, dtype={U8: torch.uint8, S8: torch.int8, U16: torch.uint16, S16: torch.int16}[out_dtype],
                                  device=x.device)
        self._chk(self.lib.qtz_quantize_tensor(self.h, _ptr(x), o, a, i, _np(params), out_dtype,
                                               int(restrict_range), _ptr(out), _stream()), "qtz_quantize_tensor")
        return out

    def dequantize(self, q, params, axis=None, in_dtype=None, shape=None, out=None):
        _check_dev(q, out)
        if in_dtype is None:
            in_dtype = {torch.uint8: U8, torch.int8: S8, torch.int32: S32, torch.uint16: U16,
                        torch.int16: S16}[q.dtype]                                    # packed 4-bit: pass in_dtype
        shape = tuple(q.shape) if shape is None else tuple(shape)
        params = np.ascontiguousarray(np.atleast_1d(params), dtype=QPARAMS)
        o, a, i = _view(shape, axis)
        assert params.shape[0] == a
        if out is None:
            out = torch.empty(shape, dtype=torch.float32, device=q.device)
        self._chk(self.lib.qtz_dequantize(self.h, _ptr(q), in_dtype, o, a, i, _np(params), _ptr(out), _stream()),
                  "qtz_dequantize")
        return out

    def simquant(self, x, params, axis=None, code_dtype=U8, restrict_range=False, out=None):
        """SimQuant (Section 2.4): quantize then de-quantize, fp32 in and out."""
        _check_dev(x, out)
        assert x.dtype == torch.float32
        params = np.ascontiguousarray(np.atleast_1d(params), dtype=QPARAMS)
        o, a, i = _view(x.shape, axis)
        assert params.shape[0] == a
        if out is None:
            out = torch.empty_like(x)
        self._chk(self.lib.qtz_simquant(self.h, _ptr(x), o, a, i, _np(params), code_dtype, int(restrict_range),
                                        _ptr(out), _stream()), "qtz_simquant")
        return out

    def sqnr(self, w, w_hat, axis=None):
        """SQNR in dB (Appendix A) per index of `axis`, or of the whole tensor."""
        _check_dev(w, w_hat)
        assert w.dtype == torch.float32 and w_hat.dtype == torch.float32 and w.shape == w_hat.shape
        o, a, i = _view(w.shape, axis)
        out = np.zeros(a, np.float64)
        self._chk(self.lib.qtz_sqnr(self.h, _ptr(w), _ptr(w_hat), o, a, i, _np(out), _stream()), "qtz_sqnr")
        return out

    def rescale_u8(self, x, x_zp, mult, rshift, y_zp, act_min=0, act_max=255, c=None, out=None, out_offset=0):
        """uint8 tensor to another quantizer (concat, Section 3.2.1); with `out`, fills the channel
        slice [out_offset, out_offset + c) of that wider tensor."""
        _check_dev(x, out)
        xp = x.shape[-1]
        c = xp if c is None else c
        if out is None:
            out = torch.zeros_like(x)
        yp = out.shape[-1]
        dst = c_void_p(out.data_ptr() + out_offset)
        self._chk(self.lib.qtz_rescale_u8(self.h, _ptr(x), x_zp, mult, rshift, dst, y_zp, act_min, act_max,
                                          x.numel() // xp, c, xp, yp, _stream()), "qtz_rescale_u8")
        return out

    def pack_u4(self, x, c=None, out=None):
        """One 4-bit code per byte [..., pitch] -> two per byte [..., (c + 1) // 2 rounded up to 16]."""
        _check_dev(x, out)
        xp = x.shape[-1]
        c = xp if c is None else c
        if out is None:
            out = torch.zeros(x.shape[:-1] + (((c + 1) // 2 + 15) // 16 * 16,), dtype=torch.uint8, device=x.device)
        self._chk(self.lib.qtz_pack_u4(self.h, _ptr(x), x.numel() // xp, c, xp, _ptr(out), out.shape[-1], _stream()),
                  "qtz_pack_u4")
        return out

    def unpack_u4(self, x, c, out=None):
        _check_dev(x, out)
        xp = x.shape[-1]
        if out is None:
            out = torch.zeros(x.shape[:-1] + ((c + 15) // 16 * 16,), dtype=torch.uint8, device=x.device)
        self._chk(self.lib.qtz_unpack_u4(self.h, _ptr(x), x.numel() // xp, c, xp, _ptr(out), out.shape[-1], _stream()),
                  "qtz_unpack_u4")
        return out

    def fold_batchnorm(self, w, conv_bias, gamma, beta, mean, var, eps):
        _check_dev(w, conv_bias, gamma, beta, mean, var)
        n = w.shape[0]
        k = w.numel() // n
        w_inf = torch.empty_like(w)
        bias_inf = torch.empty(n, dtype=torch.float32, device=w.device)
        self._chk(self.lib.qtz_fold_batchnorm(self.h, _ptr(w), _ptr(conv_bias), _ptr(gamma), _ptr(beta), _ptr(mean),
                                              _ptr(var), float(eps), n, k, _ptr(w_inf), _ptr(bias_inf), _stream()),
                  "qtz_fold_batchnorm")
        return w_inf, bias_inf

    def quantize_bias(self, bias, x_scale, w_params, per_layer=False):
        _check_dev(bias)
        w_params = np.ascontiguousarray(np.atleast_1d(w_params), dtype=QPARAMS)
        n = bias.numel()
        out = torch.empty(n, dtype=torch.int32, device=bias.device)
        self._chk(self.lib.qtz_quantize_bias(self.h, _ptr(bias), n, float(x_scale), _np(w_params), int(per_layer),
                                             _ptr(out), _stream()), "qtz_quantize_bias")
        return out

    def conv_create(self, desc: ConvDesc, w_q, bias_q=None, w_zero_point=None, mult=None, rshift=None,
                    depthwise=False):
        _check_dev(w_q, bias_q)
        zw = None if w_zero_point is None else np.array([w_zero_point], np.int32)
        m = None if mult is None else np.ascontiguousarray(mult, dtype=np.int32)
        r = None if rshift is None else np.ascontiguousarray(rshift, dtype=np.int32)
        plan = c_void_p()
        self._chk(self.lib.qtz_conv_create(self.h, byref(desc), int(depthwise), _ptr(w_q), _ptr(bias_q), _np(zw),
                                           _np(m), _np(r), byref(plan), _stream()), "qtz_conv_create")
        return ConvPlan(self, plan, desc, depthwise)

    # ---- serving: 4-bit linear layers and the 8-bit key/value cache ----
    def quantize_groups(self, w, group, dtype=torch.bfloat16, symmetric=True):
        """4-bit codes of w [n][k] (fp32) with one scale per row and `group` columns: (codes, scales, zeros) as
        linear_create takes them; zeros is None for the symmetric quantizer.  Each scale is rounded to `dtype` before
        the codes are taken with it, so that the codes belong to the scale that the layer multiplies by."""
        _check_dev(w)
        n, k = w.shape
        groups = -(-k // group)
        if groups * group != k:                       # a short last group: the zeros that fill it change no range
            w = torch.nn.functional.pad(w, (0, groups * group - k))
        w = w.reshape(n * groups, group)
        params = self.calibrate_minmax(w, axis=0, bits=4, symmetric=symmetric)
        scales = torch.from_numpy(params["scale"].copy()).to(dtype).clamp(min=torch.finfo(dtype).tiny)
        params["scale"] = scales.float().numpy()
        codes = self.quantize_tensor(w, params, axis=0, out_dtype=S4_PACKED if symmetric else U4_PACKED)
        codes = codes.reshape(n, groups * group // 2)[:, :(k + 1) // 2].contiguous()
        zeros = None if symmetric else torch.from_numpy(params["zero_point"].astype(np.uint8)).reshape(n, groups).to(w.device)
        return codes, scales.reshape(n, groups).to(w.device), zeros

    def linear_create(self, codes, scales, k, group, zeros=None, bias=None, signed=None):
        """Plan of y = x W^T + bias with packed 4-bit codes [n][(k + 1) // 2], scales [n][ceil(k / group)] and, for unsigned
        codes, zero points of the same shape.  `signed` defaults to whether there are no zero points."""
        n = codes.shape[0]
        if k <= 0 or group <= 0:
            raise ValueError("k and group are positive")
        _check_flat(self.device, torch.uint8, codes, *(() if zeros is None else (zeros,)))
        if scales.dtype not in (torch.float16, torch.bfloat16):
            raise ValueError("scales are float16 or bfloat16: the type of the layer")
        _check_flat(self.device, scales.dtype, scales, *(() if bias is None else (bias,)))
        shape = (n, -(-int(k) // int(group)))
        if codes.shape != (n, (k + 1) // 2) or scales.shape != shape or (zeros is not None and zeros.shape != shape) or \
                (bias is not None and bias.shape != (n,)):
            raise ValueError("shapes of codes, scales, zeros and bias do not belong together")
        signed = zeros is None if signed is None else signed
        desc = LinearDesc(n, int(k), int(group), S4_PACKED if signed else U4_PACKED, FTYPES[scales.dtype])
        plan = c_void_p()
        self._chk(self.lib.qtz_linear_create(self.h, byref(desc), _ptr(codes), _ptr(scales), _ptr(zeros), _ptr(bias), byref(plan),
                                             _raw_stream(self.device)), "qtz_linear_create")
        return LinearPlan(self, plan, desc, scales.dtype)

    # ---- serving: 8-bit floating point, scales for blocks of 128 ----
    def _f8_refuse(self, dtype, shape, *ts):
        """Raises for the first tensor that is not rows of neighbouring values of that type and shape on this device."""
        for t in ts:
            if t is not None and (t.dtype is not dtype or t.get_device() != self.device or t.shape != shape or (t.stride(1) != 1 and shape[1] > 1)):
                raise ValueError(f"expected rows of {dtype} values of shape {tuple(shape)} on cuda:{self.device}, got {t.dtype}, {tuple(t.shape)}, "
                                 f"strides {t.stride()} on {t.device}")

    def f8_rmsnorm(self, x, gain, eps=1e-6, residual=None, codes=True, values=False, sum_out=None):
        """Root-mean-square norm of the rows of x (+ residual) [rows][k]: (codes, scales, values, sum).  codes and scales (e4m3
        [rows][k], fp32 [rows][ceil(k / 128)]) are None unless `codes`, values (the type of x) unless `values`, sum (x + residual)
        without a residual.  `sum_out` may be `residual` itself."""
        dtype, shape, device = x.dtype, x.shape, self.device
        ftype = FTYPES.get(dtype)
        if ftype is None or len(shape) != 2:
            raise ValueError("expected rows of float32, float16 or bfloat16 values")
        rows, k = shape
        total, r_at, r_stride, t_at, t_stride = None, None, 0, None, 0
        if residual is not None:
            total = sum_out
            if total is None:
                t_stride = (k + 15) // 16 * 16
                total = x.new_empty_strided(shape, (t_stride, 1))
                self._f8_refuse(dtype, shape, x, residual)
            else:
                self._f8_refuse(dtype, shape, x, residual, total)
                t_stride = total.stride(0)
            r_at, r_stride, t_at = residual.data_ptr(), residual.stride(0), total.data_ptr()
        else:
            if sum_out is not None:
                raise ValueError("sum_out belongs to a residual")
            self._f8_refuse(dtype, shape, x)
        if gain.dtype is not dtype or gain.shape != (k,) or gain.get_device() != device or not gain.is_contiguous():
            raise ValueError(f"expected a gain of {k} {dtype} values on cuda:{device}")
        out = q = scales = None
        v_at, v_stride, q_at, q_stride, s_at = None, 0, None, 0, None
        blocks = (k + 127) // 128
        if values:
            v_stride = (k + 15) // 16 * 16
            out = x.new_empty_strided(shape, (v_stride, 1))
            v_at = out.data_ptr()
        if codes:
            q_stride = (k + 31) // 32 * 32                # 16 bytes are asked for; whole sectors are written faster
            q, scales = x.new_empty_strided(shape, (q_stride, 1), dtype=E4M3), x.new_empty((rows, blocks), dtype=torch.float32)
            q_at, s_at = q.data_ptr(), scales.data_ptr()
        rc = self.lib.qtz_f8_rmsnorm(self.h, x.data_ptr(), x.stride(0), r_at, r_stride, gain.data_ptr(), eps, rows, k, ftype, t_at, t_stride, v_at, v_stride,
                                     q_at, q_stride, s_at, blocks, _raw_stream(device))
        if rc:
            self._chk(rc, "qtz_f8_rmsnorm")
        return q, scales, out, total

    def f8_quantize(self, x, gate=None):
        """Codes (e4m3 [rows][k]) and scales (fp32 [rows][ceil(k / 128)]) of x [rows][k], or of silu(gate) * x."""
        dtype, shape = x.dtype, x.shape
        ftype = FTYPES.get(dtype)
        if ftype is None or len(shape) != 2:
            raise ValueError("expected rows of float32, float16 or bfloat16 values")
        self._f8_refuse(dtype, shape, x, gate)
        rows, k = shape
        pitch, blocks = (k + 31) // 32 * 32, (k + 127) // 128
        q, scales = x.new_empty_strided(shape, (pitch, 1), dtype=E4M3), x.new_empty((rows, blocks), dtype=torch.float32)
        g_at, g_stride = (None, 0) if gate is None else (gate.data_ptr(), gate.stride(0))
        rc = self.lib.qtz_f8_quantize(self.h, x.data_ptr(), x.stride(0), g_at, g_stride, rows, k, ftype, q.data_ptr(), pitch, scales.data_ptr(), blocks,
                                      _raw_stream(self.device))
        if rc:
            self._chk(rc, "qtz_f8_quantize")
        return q, scales

    def f8_quantize_weights(self, w):
        """Codes (e4m3 [n][k]) and scales (fp32 [ceil(n / 128)][ceil(k / 128)]) of weights w [n][k], as f8_linear_create takes them."""
        if w.dim() != 2 or w.dtype not in FTYPES:
            raise ValueError("expected a matrix of float32, float16 or bfloat16 values")
        self._f8_refuse(w.dtype, w.shape, w)
        n, k = w.shape
        codes = torch.empty((n, k), dtype=E4M3, device=w.device)
        scales = torch.empty((-(-n // 128), -(-k // 128)), dtype=torch.float32, device=w.device)
        self._chk(self.lib.qtz_f8_quantize_weights(self.h, _ptr(w), w.stride(0), n, k, FTYPES[w.dtype], _ptr(codes), _ptr(scales),
                                                   _raw_stream(self.device)), "qtz_f8_quantize_weights")
        return codes, scales

    def f8_linear_create(self, codes, scales, bias=None):
        """Plan of y = x W^T + bias with e4m3 codes of W [n][k] and fp32 scales [ceil(n / 128)][ceil(k / 128)]."""
        if codes.dim() != 2:
            raise ValueError("expected codes [n][k]")
        n, k = codes.shape
        self._f8_refuse(E4M3, codes.shape, codes)
        _check_flat(self.device, torch.float32, scales)
        if scales.shape != (-(-n // 128), -(-k // 128)):
            raise ValueError(f"expected a scale for each 128 x 128 block of [{n}][{k}], got {tuple(scales.shape)}")
        if bias is not None:
            _check_flat(self.device, bias.dtype, bias)
            if bias.shape != (n,) or bias.dtype not in FTYPES:
                raise ValueError(f"expected a bias of {n} values")
        plan = c_void_p()
        self._chk(self.lib.qtz_f8_linear_create(self.h, n, k, _ptr(codes), codes.stride(0), _ptr(scales), _ptr(bias),
                                                F32 if bias is None else FTYPES[bias.dtype], byref(plan), _raw_stream(self.device)), "qtz_f8_linear_create")
        return F8LinearPlan(self, plan, n, k)

    def kv_schedule(self, cached, added, table, free, free_count, block_tokens, capacity):
        """qtz_kv_schedule: writes the new blocks into `table` and returns (starts, lens, slots, report)."""
        device = self.device
        _check_flat(device, torch.int32, cached, added, table, free, free_count)
        b, (rows, width) = cached.numel(), table.shape
        if added.numel() != b or rows != b or free_count.numel() != 1:
            raise ValueError("cached, added and table describe different numbers of requests")
        slots = cached.new_empty(capacity, dtype=torch.int64)
        starts, lens, report = cached.new_empty(2 * b + 5).split_with_sizes((b + 1, b, 4))
        at = starts.data_ptr()
        rc = self.lib.qtz_kv_schedule(self.h, cached.data_ptr(), added.data_ptr(), b, block_tokens, table.data_ptr(), width, free.data_ptr(),
                                      free_count.data_ptr(), at, at + 4 * (b + 1), slots.data_ptr(), capacity, at + 4 * (2 * b + 1),
                                      _raw_stream(device))
        if rc:
            self._chk(rc, "qtz_kv_schedule")
        return starts, lens, slots, report

    def kv_cache(self, blocks, kv_heads, block_tokens, head_dim):
        """A cache whose memory torch owns, every block all zero."""
        device = f"cuda:{self.device}"
        k, v = (torch.zeros(blocks, kv_heads, block_tokens, head_dim, dtype=torch.int8, device=device) for _ in range(2))
        ks, vs = (torch.full((blocks, kv_heads), 2.0 ** -100, device=device) for _ in range(2))
        return KvCache(self, k, v, ks, vs)

    def add_u8(self, a, a_zp, a_mult, b, b_zp, b_mult, rshift, y_zp, act_min, act_max, c, out=None):
        _check_dev(a, b, out)
        pitch = a.shape[-1]
        pixels = a.numel() // pitch
        out = torch.empty_like(a) if out is None else out
        self._chk(self.lib.qtz_add_u8(self.h, _ptr(a), a_zp, a_mult, _ptr(b), b_zp, b_mult, rshift, _ptr(out), y_zp,
                                      act_min, act_max, pixels, c, pitch, _stream()), "qtz_add_u8")
        return out

    def maxpool_u8(self, x, c, k, stride, pad, out=None):
        _check_dev(x, out)
        b, hh, ww, pitch = x.shape
        oh, ow = (hh + 2 * pad - k) // stride + 1, (ww + 2 * pad - k) // stride + 1
        out = torch.empty((b, oh, ow, pitch), dtype=torch.uint8, device=x.device) if out is None else out
        self._chk(self.lib.qtz_maxpool_u8(self.h, _ptr(x), _ptr(out), b, hh, ww, c, pitch, k, stride, pad, _stream()),
                  "qtz_maxpool_u8")
        return out

    def global_avgpool_u8(self, x, x_zp, y_zp, mult, rshift, c, out=None):
        _check_dev(x, out)
        b, hh, ww, pitch = x.shape
        out = torch.empty((b, 1, 1, pitch), dtype=torch.uint8, device=x.device) if out is None else out
        self._chk(self.lib.qtz_global_avgpool_u8(self.h, _ptr(x), x_zp, _ptr(out), y_zp, mult, rshift, b, hh * ww, c,
                                                 pitch, _stream()), "qtz_global_avgpool_u8")
        return out


class ConvPlan:
    """Owns a qtz_conv_plan."""

    def __init__(self, handle: Handle, plan, desc: ConvDesc, depthwise: bool):
        self.handle, self.plan, self.desc, self.depthwise = handle, plan, desc, bool(depthwise)
        d = desc
        self.oh = (d.h + 2 * d.pad - d.kh) // d.stride + 1
        self.ow = (d.w + 2 * d.pad - d.kw) // d.stride + 1

    @property
    def kernel(self) -> str:
        return self.handle.lib.qtz_conv_plan_kernel(self.plan).decode()

    @property
    def detail(self) -> str:
        return self.handle.lib.qtz_conv_plan_detail(self.plan).decode()

    def empty_output(self, device):
        d = self.desc
        if d.outkind == OUT_S32_RAW:
            return torch.empty((d.batch, self.oh, self.ow, d.n), dtype=torch.int32, device=device)
        return torch.empty((d.batch, self.oh, self.ow, d.c_pitch_out), dtype=torch.uint8, device=device)

    def __call__(self, x, x_zero_point, y_zero_point=0, act_min=0, act_max=255, out=None):
        _check_dev(x, out)
        out = self.empty_output(x.device) if out is None else out
        fn = self.handle.lib.qtz_depthwise_u8 if self.depthwise else self.handle.lib.qtz_conv2d_u8
        self.handle._chk(fn(self.plan, _ptr(x), int(x_zero_point), _ptr(out), int(y_zero_point), int(act_min),
                            int(act_max), _stream()), "qtz_depthwise_u8" if self.depthwise else "qtz_conv2d_u8")
        return out

    def add_fused(self, x, x_zero_point, residual: Residual, s, y_zero_point, act_min, act_max, out=None):
        """qtz_conv2d_add_u8: this convolution and the element-wise add with `s` in one kernel."""
        _check_dev(x, s, out)
        out = self.empty_output(x.device) if out is None else out
        self.handle._chk(self.handle.lib.qtz_conv2d_add_u8(self.plan, _ptr(x), int(x_zero_point), byref(residual), _ptr(s),
                                                           _ptr(out), int(y_zero_point), int(act_min), int(act_max), _stream()),
                         "qtz_conv2d_add_u8")
        return out

    def after_depthwise(self, dw_plan, x, x_zero_point, mid_zero_point, mid_act_min, mid_act_max, y_zero_point, act_min,
                        act_max, out=None):
        """qtz_conv2d_dw_pw_u8: the 3x3 depthwise plan `dw_plan` and this pointwise plan in one kernel.  Raises
        QtzError (code ERR_UNSUPPORTED) when the pair cannot run fused."""
        _check_dev(x, out)
        out = self.empty_output(x.device) if out is None else out
        self.handle._chk(self.handle.lib.qtz_conv2d_dw_pw_u8(dw_plan.plan, self.plan, _ptr(x), int(x_zero_point),
                                                             int(mid_zero_point), int(mid_act_min), int(mid_act_max), _ptr(out),
                                                             int(y_zero_point), int(act_min), int(act_max), _stream()),
                         "qtz_conv2d_dw_pw_u8")
        return out

    def set_profile_events(self, start=None, stop=None):
        """start/stop: torch.cuda.Event(enable_timing=True) already created (recorded once), or None."""
        s = None if start is None else c_void_p(start.cuda_event)
        e = None if stop is None else c_void_p(stop.cuda_event)
        self.handle._chk(self.handle.lib.qtz_conv_set_profile_events(self.plan, s, e), "qtz_conv_set_profile_events")

    def close(self):
        if self.plan:
            self.handle.lib.qtz_conv_destroy(self.plan)
            self.plan = c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class LinearPlan:
    """Owns a qtz_linear_plan: y = x W^T + bias with 4-bit weights."""

    def __init__(self, handle: Handle, plan, desc: LinearDesc, dtype):
        self.handle, self.plan, self.desc, self.dtype, self.device = handle, plan, desc, dtype, handle.device
        self.n, self.k, self.k_up = desc.n, desc.k, (desc.k + 7) // 8 * 8
        self._run = handle.lib.qtz_linear_w4

    def __call__(self, x, out=None):
        """x [rows][k] (or more leading axes that fold into rows); rows may lie apart by a multiple of 16 bytes."""
        n, k, dtype = self.n, self.k, self.dtype
        lead = x.shape[:-1]
        if x.shape[-1] != k or x.stride(-1) != 1:
            raise ValueError(f"expected rows of {k} neighbouring values, got {tuple(x.shape)} with strides {x.stride()}")
        if x.dtype is not dtype or x.get_device() != self.device:
            raise ValueError(f"expected {dtype} on cuda:{self.device}, got {x.dtype} on {x.device}")
        if len(lead) != 1:
            x = x.view(-1, k)
        rows = x.shape[0]
        if out is None:
            y = x.new_empty((rows, n))
            out = y if len(lead) == 1 else y.view(*lead, n)
        else:
            _check_on(self.device, dtype, out)
            if out.shape != lead + (n,) or out.stride(-1) != 1:
                raise ValueError("out has another shape")
            y = out if len(lead) == 1 else out.view(-1, n)
        if not self.handle.h:
            raise ValueError("the handle of this plan is closed")
        # a single row has no stride to keep: torch reports any value for it
        if rows == 1:
            rc = self._run(self.plan, x.data_ptr(), self.k_up, 1, y.data_ptr(), n, _raw_stream(self.device))
        else:
            rc = self._run(self.plan, x.data_ptr(), x.stride(0), rows, y.data_ptr(), y.stride(0), _raw_stream(self.device))
        if rc:
            self.handle._chk(rc, "qtz_linear_w4")
        return out

    def close(self):
        if self.plan:
            self.handle.lib.qtz_linear_destroy(self.plan)
            self.plan = c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class F8LinearPlan:
    """Owns a qtz_f8_linear_plan: y = x W^T + bias with e4m3 activations and weights."""

    def __init__(self, handle: Handle, plan, n, k):
        self.handle, self.plan, self.n, self.k, self.device, self.blocks = handle, plan, n, k, handle.device, -(-k // 128)
        self._run = handle.lib.qtz_f8_linear

    def __call__(self, codes, scales, dtype=torch.bfloat16, out=None):
        """codes [rows][k] in e4m3 (rows a multiple of 16 bytes apart), scales [rows][ceil(k / 128)] in fp32 with any strides."""
        device, n, shape, (stride, next_to), (row_stride, block_stride) = self.device, self.n, codes.shape, codes.stride(), scales.stride()
        if codes.dtype is not E4M3 or codes.get_device() != device or scales.dtype is not torch.float32 or scales.get_device() != device:
            raise ValueError(f"expected {E4M3} codes and float32 scales on cuda:{device}, got {codes.dtype} on {codes.device}, {scales.dtype} on {scales.device}")
        rows, k = shape
        if k != self.k or (next_to != 1 and k > 1) or scales.shape != (rows, self.blocks):
            raise ValueError(f"expected rows of {self.k} neighbouring codes and {self.blocks} scales, got {tuple(shape)} with strides {codes.stride()} "
                             f"and {tuple(scales.shape)}")
        if out is None:
            ftype, y_stride = FTYPES.get(dtype), n
            if ftype is None:
                raise ValueError("y is float32, float16 or bfloat16")
            out = codes.new_empty((rows, n), dtype=dtype)
        else:
            ftype = FTYPES.get(out.dtype)
            if ftype is None or out.shape != (rows, n) or (out.stride(1) != 1 and n > 1) or out.get_device() != device:
                raise ValueError(f"expected out of shape {(rows, n)} on cuda:{device}")
            y_stride = out.stride(0)
        if not self.handle.h:
            raise ValueError("the handle of this plan is closed")
        rc = self._run(self.plan, codes.data_ptr(), stride, scales.data_ptr(), row_stride, block_stride, rows, out.data_ptr(), y_stride, ftype,
                       _raw_stream(device))
        if rc:
            self.handle._chk(rc, "qtz_f8_linear")
        return out

    def close(self):
        if self.plan:
            self.handle.lib.qtz_f8_linear_destroy(self.plan)
            self.plan = c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class KvCache:
    """A paged 8-bit key/value cache in torch tensors: codes [blocks][kv_heads][block_tokens][head_dim] int8, scales
    [blocks][kv_heads] fp32.  attention() keeps its workspace here: one stream at a time."""

    def __init__(self, handle: Handle, k, v, k_scale, v_scale):
        _check_flat(handle.device, torch.int8, k, v)
        _check_flat(handle.device, torch.float32, k_scale, v_scale)
        if k.dim() != 4 or v.shape != k.shape or k_scale.shape != k.shape[:2] or v_scale.shape != k.shape[:2]:
            raise ValueError("shapes of codes and scales do not belong together")
        self.handle, self.k, self.v, self.k_scale, self.v_scale = handle, k, v, k_scale, v_scale
        self.blocks, self.kv_heads, self.block_tokens, self.head_dim = k.shape
        self._desc = KvCacheDesc(k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), *k.shape)
        self._ref = byref(self._desc)
        self.device, self.lib, self.scale = handle.device, handle.lib, self.head_dim ** -0.5
        # zero-filled here, not by the first call of attention(), whose fill a graph that captures it would keep for itself
        size = self.lib.qtz_kv_attention_workspace_bytes(handle.h, self._ref)
        self.workspace = torch.zeros(max(size, 16), dtype=torch.uint8, device=k.device)
        handle._caches.add(self)

    def reset_workspace(self):
        """Zero-fills the workspace of attention() on the current stream: a call that gave up may have left parts counted in it.
        Handle.device_status() does so when it reports a timeout."""
        self.workspace.zero_()

    def append(self, k, v, slots):
        """Quantizes new keys and values [tokens][kv_heads][head_dim] (any token and head stride) into `slots`."""
        dev, dtype, shape = self.device, k.dtype, (slots.numel(), self.kv_heads, self.head_dim)
        _check_flat(dev, torch.int64, slots)
        _check_on(dev, dtype, k, v)
        ks, vs = k.stride(), v.stride()
        if k.shape != shape or v.shape != shape or ks[2] != 1 or vs[2] != 1 or dtype not in FTYPES:
            raise ValueError(f"expected keys and values of shape {shape}")
        rc = self.lib.qtz_kv_append(self.handle.h, self._ref, k.data_ptr(), ks[0], ks[1], v.data_ptr(), vs[0], vs[1], FTYPES[dtype],
                                    slots.data_ptr(), shape[0], _raw_stream(dev))
        if rc:
            self.handle._chk(rc, "qtz_kv_append")

    def read(self, slots, dtype=torch.float32):
        """Real values of the slots: keys and values [tokens][kv_heads][head_dim]."""
        dev, tokens = self.device, slots.numel()
        _check_flat(dev, torch.int64, slots)
        k, v = slots.new_empty((2, tokens, self.kv_heads, self.head_dim), dtype=dtype).unbind(0)
        rc = self.lib.qtz_kv_read(self.handle.h, self._ref, slots.data_ptr(), tokens, FTYPES.get(dtype, -1), k.data_ptr(), v.data_ptr(),
                                  _raw_stream(dev))
        if rc:
            self.handle._chk(rc, "qtz_kv_read")
        return k, v

    def attention(self, q, starts, lens, table, scale=None, window=0, out=None, return_lse=False):
        """q [tokens][q_heads][head_dim] of the requests' newest tokens (rows starts[r] .. starts[r + 1]); returns y, or (y, lse)."""
        dev, dtype, shape = self.device, q.dtype, q.shape
        _check_on(dev, dtype, q)
        _check_flat(dev, torch.int32, starts, lens, table)
        b, (rows, width), qs = lens.numel(), table.shape, q.stride()
        if len(shape) != 3 or shape[2] != self.head_dim or qs[2] != 1 or dtype not in FTYPES:
            raise ValueError(f"expected queries [tokens][heads][{self.head_dim}]")
        if starts.numel() != b + 1 or rows != b:
            raise ValueError("starts, lens and table describe different numbers of requests")
        if out is None:
            out = q.new_empty(shape)
        else:
            _check_on(dev, dtype, out)
            if out.shape != shape or out.stride(2) != 1:
                raise ValueError("out has another shape")
        lse = q.new_empty(shape[:2], dtype=torch.float32) if return_lse else None
        ys = out.stride()
        rc = self.lib.qtz_kv_attention(self.handle.h, self._ref, q.data_ptr(), qs[0], qs[1], shape[1], FTYPES[dtype], starts.data_ptr(), lens.data_ptr(), b,
                                       shape[0], table.data_ptr(), width, self.scale if scale is None else scale, window, out.data_ptr(), ys[0],
                                       ys[1], lse.data_ptr() if return_lse else None, self.workspace.data_ptr(), _raw_stream(dev))
        if rc:
            self.handle._chk(rc, "qtz_kv_attention")
        return (out, lse) if return_lse else out


def conv_desc(batch, h, w, c, n, kh, kw, stride, pad, wkind=W_S8_PER_CHANNEL_SYM, outkind=OUT_U8,
              c_pitch_in=None, c_pitch_out=None) -> ConvDesc:
    rup = lambda v: (v + 15) // 16 * 16
    return ConvDesc(batch, h, w, c, rup(c) if c_pitch_in is None else c_pitch_in, n,
                    rup(n) if c_pitch_out is None else c_pitch_out, kh, kw, stride, pad, wkind, outkind)
