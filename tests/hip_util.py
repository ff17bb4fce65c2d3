"""Device memory, streams and graphs for tests that call single operations (``ooc.run_fn``), through
the HIP runtime the library itself is linked to.  Every array sits between guard bytes, so a write
outside it shows."""

import ctypes

import numpy as np

from paper_2010_14109_amd import ooc

_hip = None
GUARD = 4096
PATTERN = 0xA5


def hip():
    global _hip
    if _hip is None:
        ooc.load()
        path = next(line.split()[-1] for line in open("/proc/self/maps") if "libamdhip64" in line)
        _hip = ctypes.CDLL(path)
    return _hip


def check(status, what):
    if status != 0:
        hip().hipGetErrorString.restype = ctypes.c_char_p
        raise RuntimeError(f"{what}: {hip().hipGetErrorString(status).decode()}")


class Array:
    """A NumPy array's copy on the device; ``get`` copies it back and looks at the guards."""

    def __init__(self, a):
        a = np.ascontiguousarray(a)
        self.shape, self.dtype, self.nbytes = a.shape, a.dtype, a.nbytes
        whole = np.full(self.nbytes + 2 * GUARD, PATTERN, np.uint8)
        whole[GUARD:GUARD + self.nbytes] = a.reshape(-1).view(np.uint8)
        p = ctypes.c_void_p()
        check(hip().hipMalloc(ctypes.byref(p), ctypes.c_size_t(whole.nbytes)), "hipMalloc")
        self.base = p.value
        self.ptr = self.base + GUARD
        check(hip().hipMemcpy(p, whole.ctypes.data_as(ctypes.c_void_p),
                              ctypes.c_size_t(whole.nbytes), 1), "hipMemcpy to the device")

    def get(self):
        whole = np.empty(self.nbytes + 2 * GUARD, np.uint8)
        check(hip().hipMemcpy(whole.ctypes.data_as(ctypes.c_void_p), ctypes.c_void_p(self.base),
                              ctypes.c_size_t(whole.nbytes), 2), "hipMemcpy to the host")
        assert (whole[:GUARD] == PATTERN).all() and (whole[-GUARD:] == PATTERN).all(), \
            "written outside the array"
        return whole[GUARD:GUARD + self.nbytes].view(self.dtype).reshape(self.shape).copy()

    def __del__(self):
        if getattr(self, "base", None):
            hip().hipFree(ctypes.c_void_p(self.base))


def synchronize():
    check(hip().hipDeviceSynchronize(), "hipDeviceSynchronize")


class Stream:
    def __init__(self):
        p = ctypes.c_void_p()
        check(hip().hipStreamCreateWithFlags(ctypes.byref(p), 1), "hipStreamCreate")
        self.ptr = p.value

    def __del__(self):
        if getattr(self, "ptr", None):
            hip().hipStreamDestroy(ctypes.c_void_p(self.ptr))

    def record(self, calls, mode=2):
        """A graph of what ``calls()`` enqueues on this stream, as a function that replays it.
        ``mode``: hipStreamCaptureMode (0 global, 2 relaxed)."""
        s, graph, run = ctypes.c_void_p(self.ptr), ctypes.c_void_p(), ctypes.c_void_p()
        check(hip().hipStreamBeginCapture(s, mode), "hipStreamBeginCapture")
        try:
            calls()
        finally:
            status = hip().hipStreamEndCapture(s, ctypes.byref(graph))
        check(status, "hipStreamEndCapture")
        check(hip().hipGraphInstantiate(ctypes.byref(run), graph, None, None, ctypes.c_size_t(0)),
              "hipGraphInstantiate")

        def replay():
            check(hip().hipGraphLaunch(run, s), "hipGraphLaunch")
        return replay


def call(op, arrays, access, attrs, stream=None):
    ooc.run_fn(op, [(a.ptr, a.nbytes) for a in arrays], access, attrs,
               stream=stream.ptr if stream else 0)


def empty(shape, dtype=np.float32):
    """Output memory, filled with NaN (0x7f for integers), so that an entry left out shows."""
    a = np.empty(shape, dtype)
    a.fill(np.nan if np.issubdtype(dtype, np.floating) else 0x7f)
    return Array(a)
