"""Arrays in device memory for the operators' tests: the HIP runtime that the library is linked with, through ctypes, behind the
few attributes the binding reads."""
import ctypes
from types import SimpleNamespace

import numpy as np

import paper_2505_21594_amd as ee

_hip = None


def hip():
    global _hip
    if _hip is None:
        ee.load_library()
        _hip = ctypes.CDLL("libamdhip64.so.7")
        _hip.hipMalloc.argtypes = [ctypes.POINTER(ctypes.c_void_p), ctypes.c_size_t]
        _hip.hipFree.argtypes = [ctypes.c_void_p]
        _hip.hipMemcpy.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int]
        for name in ("hipStreamCreate", "hipStreamSynchronize", "hipStreamDestroy", "hipStreamBeginCapture", "hipStreamEndCapture", "hipGraphInstantiate",
                     "hipGraphLaunch", "hipGraphExecDestroy", "hipGraphDestroy"):
            getattr(_hip, name).restype = ctypes.c_int
    return _hip


def ok(rc):
    assert rc == 0, f"HIP error {rc}"


def bf16_bits(x):
    """float32 -> bf16 bits, to nearest even; NaN stays NaN."""
    x = np.ascontiguousarray(x, np.float32)
    u = x.view(np.uint32).astype(np.uint64)
    r = ((u + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint16)
    return np.where(np.isnan(x), np.uint16(0x7FC0), r)


def bf16_values(bits):
    return (np.asarray(bits, np.uint16).astype(np.uint32) << 16).view(np.float32)


NAMES = {np.dtype(np.float32): "float32", np.dtype(np.float16): "float16", np.dtype(np.int32): "int32", np.dtype(np.uint8): "uint8", np.dtype(np.uint16): "bfloat16"}


class Dev:
    """A device array; uint16 stands for bf16.  `view(...)`: another shape or strides on the same memory."""

    def __init__(self, a, shape=None, strides=None, offset=0, base=None):
        if base is None:
            a = np.ascontiguousarray(a)
            self._p = ctypes.c_void_p()
            self._n = max(a.nbytes, 16)
            if on_gpu():
                ok(hip().hipMalloc(ctypes.byref(self._p), self._n))
                if a.nbytes:
                    ok(hip().hipMemcpy(self._p, a.ctypes.data, a.nbytes, 1))
            else:
                self._p.value = 1 << 20   # argument checks run without a GPU
            self._np, self._owner, self._base = a.dtype, True, None
            shape, strides = a.shape, tuple(s // a.itemsize for s in a.strides)
        else:
            self._np, self._owner, self._base, self._p = base._np, False, base, base._p
        self.shape, self._strides, self._offset = tuple(shape), tuple(strides), offset
        self.dtype, self.device = NAMES[self._np], SimpleNamespace(type="cuda", index=0)

    def data_ptr(self):
        return self._p.value + self._offset * self._np.itemsize

    def stride(self):
        return self._strides

    def view(self, shape, strides, offset=0):
        return Dev(None, shape, strides, self._offset + offset, self)

    def numpy(self):
        """The whole allocation, as the array it was made of."""
        assert self._owner
        out = np.empty(self.shape, self._np)
        ok(hip().hipDeviceSynchronize())
        if out.nbytes:
            ok(hip().hipMemcpy(out.ctypes.data, self._p, out.nbytes, 2))
        return out

    def write(self, a):
        a = np.ascontiguousarray(a, self._np)
        assert a.shape == self.shape
        ok(hip().hipMemcpy(self._p, a.ctypes.data, a.nbytes, 1))

    def __del__(self):
        if getattr(self, "_owner", False) and on_gpu() and self._p.value:
            _hip.hipFree(self._p)


_gpu = None


def on_gpu():
    global _gpu
    if _gpu is None:
        import os
        _gpu = os.path.exists("/dev/kfd")
    return _gpu


FLOATS = {"bf16": np.uint16, "fp16": np.float16, "fp32": np.float32}


def encode(x, kind):
    return bf16_bits(x) if kind == "bf16" else np.asarray(x, FLOATS[kind])


def decode(a):
    return (bf16_values(a) if a.dtype == np.uint16 else a).astype(np.float64)


HALF_STEP = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11, "fp32": 2.0 ** -24}
