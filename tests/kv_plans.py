"""How attention over the cache is cut up: csrc/kv_plan.h, compiled for the host."""
import ctypes
import os
import subprocess
import tempfile

from conftest import ROOT

SOURCE = """
#include "kv_plan.h"
using namespace nvfp4::kv;
extern "C" void plan_of(int64_t tokens, int64_t batch, int64_t max_q, int q_heads, int heads, int dim, int64_t length, int64_t prefix,
                        int64_t* out) {
    const Plan p = make_plan(Sizes{tokens, batch, max_q, q_heads, heads, dim, length, prefix});
    const int64_t v[] = {p.own.rows, p.own.tiles, p.own.parts, p.prefix.rows, p.prefix.tiles, p.prefix.parts, p.through, p.merge, p.bytes,
                         p.fits()};
    for (int i = 0; i < 10; i++) out[i] = v[i];
}
extern "C" int64_t tokens_of(int64_t length, int64_t parts, int64_t step) { return part_tokens(length, parts, step); }
extern "C" uint32_t tokens_of32(uint32_t length, uint32_t parts, uint32_t step) { return part_tokens32(length, parts, step); }
"""
NAMES = ("rows", "tiles", "parts", "prefix_rows", "prefix_tiles", "prefix_parts", "through", "merge", "bytes", "fits")
_lib = None


def lib():
    global _lib
    if _lib is None:
        with tempfile.TemporaryDirectory() as d:
            src, so = os.path.join(d, "plan.cpp"), os.path.join(d, "plan.so")
            with open(src, "w") as f:
                f.write(SOURCE)
            subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2606_07618_gb300", "csrc"),
                            src, "-o", so], check=True)
            _lib = ctypes.CDLL(so)
        i64, i = ctypes.c_int64, ctypes.c_int
        _lib.plan_of.argtypes = [i64, i64, i64, i, i, i, i64, i64, ctypes.POINTER(i64)]
        _lib.tokens_of.argtypes, _lib.tokens_of.restype = [i64] * 3, i64
        _lib.tokens_of32.argtypes, _lib.tokens_of32.restype = [ctypes.c_uint32] * 3, ctypes.c_uint32
    return _lib


def plan_of(tokens, batch, max_q, q_heads, heads, dim, length, prefix=0):
    out = (ctypes.c_int64 * 10)()
    lib().plan_of(tokens, batch, max_q, q_heads, heads, dim, length, prefix, out)
    return dict(zip(NAMES, out))


def path(p):
    """The kernel of the own pass (rows of a block), how its parts are joined, and the prefix's kernel."""
    join = "merge" if p["merge"] else "workspace" if p["through"] else "cluster" if p["parts"] > 1 else "alone"
    return p["rows"], join, p["prefix_rows"]


def path_of(s):
    """The same for a kv_reference.Setting."""
    up = lambda n: -(-n // s.page) * s.page  # noqa: E731
    return path(plan_of(s.total, len(s.lens), max(s.queries), s.heads * s.group, s.heads, s.dim, max([up(n) for n in s.lens] + [s.page]),
                        up(s.prefix)))
