"""Runs checks of tests/routed_ref.py on the kernels' CPU model: routed.py LIBRARY CASES, the cases a JSON
list of [check, arguments, keywords]. Every case runs with its arrays at the end and at the beginning of
their pages; a touched page ends the process with status 3, which names the case by what was printed last."""

import ctypes
import json
import os
import sys
import traceback

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
sys.path[:0] = [os.path.dirname(HERE), os.path.dirname(os.path.dirname(HERE))]

import routed_ref as ref  # noqa: E402
from gpu_util import bf16_bits  # noqa: E402

P, i64, i32, u32, f64 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_uint32, ctypes.c_double
NUMPY = {"f32": np.float32, "bf16": np.uint16, "i8": np.int8, "u8": np.uint8}


class Array:
    """A flat array in the model's memory, or rows of it."""

    def __init__(self, engine, a, kind=None, shape=None, ld=0, fill=None):
        self.flat = engine.take(a)
        self.ptr, self.kind, self.shape, self.ld, self.fill = self.flat.ctypes.data, kind, shape, ld, fill
        self.margin = None if shape is None else self._margin().copy()

    def _margin(self):
        n, F = self.shape
        return np.concatenate([self.flat[i * self.ld + F:(i + 1) * self.ld] for i in range(max(n - 1, 0))]
                              or [self.flat[:0]])

    def get(self):
        if self.shape is None:
            return self.flat.copy().reshape(self.view)
        n, F = self.shape
        out = np.empty((n, F), self.flat.dtype)
        for i in range(n):
            out[i] = self.flat[i * self.ld:i * self.ld + F]
        if self.kind == "bf16":
            out = (out.astype(np.uint32) << 16).view(np.float32)
        return out

    def check_margins(self):
        assert np.array_equal(self._margin(), self.margin), "written between the rows"


class Engine:
    stream = None

    def __init__(self, path):
        import paper_2411_16025_amd as pkg
        self.lib = ctypes.CDLL(path)
        for name in ("group_ids", "embed_fwd", "embed_bwd", "route_fwd", "route_bwd", "combine_fwd",
                     "combine_bwd", "pack8", "unpack8", "gemm_grouped_q8"):
            f, g = getattr(self.lib, "gcn_" + name), getattr(pkg.lib(), "gcn_" + name)
            f.argtypes, f.restype = g.argtypes, ctypes.c_int
        self.lib.model_array.argtypes, self.lib.model_array.restype = [i64], P
        self.lib.model_start()

    def error(self):
        return ""

    def take(self, a):
        a = np.ascontiguousarray(a)
        p = self.lib.model_array(a.nbytes)
        m = np.frombuffer((ctypes.c_char * a.nbytes).from_address(p), a.dtype) if a.nbytes else a.ravel()
        m[:] = a.ravel()
        return m

    def put(self, a):
        r = Array(self, a)
        r.view = np.shape(a)
        return r

    def new(self, shape, dtype):
        return self.put(np.full(shape, 77, dtype))

    def work(self, size):
        return (self.lib.model_array(size + 256) + 255) // 256 * 256 if size else None

    def rows(self, x, kind, pad=0, shift=0, fill=np.nan):
        n, F = x.shape
        if kind in ("f32", "bf16"):
            conv = (lambda v: bf16_bits(v)) if kind == "bf16" else (lambda v: np.asarray(v, np.float32))
        else:
            conv = lambda v: np.asarray(v, NUMPY[kind])  # noqa: E731
        ld = F + pad
        flat = np.empty(max((n - 1) * ld + F, 0) if n else 0, NUMPY[kind])
        if kind not in ("f32", "bf16") and fill != fill:
            fill = 77
        flat[:] = conv(np.full(1, fill, np.float32 if kind in ("f32", "bf16") else NUMPY[kind]))[0]
        for i in range(n):
            flat[i * ld:i * ld + F] = conv(np.ascontiguousarray(x[i]))
        return Array(self, flat, kind, (n, F), ld, fill)


def main():
    e = Engine(sys.argv[1])
    for name, args, kw in json.load(open(sys.argv[2])):
        for at_end in (1, 0):
            print(name, args, kw, "end" if at_end else "beginning", flush=True)
            e.lib.model_side(at_end)
            try:
                getattr(ref, name)(e, *args, **kw)
            except AssertionError:
                traceback.print_exc()
                os._exit(1)
            e.lib.model_check()
            e.lib.model_release()


main()
