"""Which kernel, tile width and split each product of a 4-bit call takes: csrc/fp4_plan.h, compiled for the host."""
import ctypes
import os
import subprocess
import tempfile

from conftest import ROOT

NV, MX, BF16 = 0, 1, 2
PLAIN, GATED, GRAD = 0, 1, 2
SMS = 152                                                        # a GB300's

SOURCE = """
#include "fp4_plan.h"
using namespace nvfp4;
extern "C" void plan_of(int kind, int mode, int f32, int64_t t, int64_t n, int64_t k, int64_t ldq, int sms, int64_t* out) {
    const mm::Sizes s = {kind, mode, f32, t, n, k, ldq};
    out[0] = mm::few_tokens(s, sms);
    if (out[0]) {
        const mm::TilePlan b = mm::tile_plan(s, sms);
        out[1] = 1 << b.log_split;
        out[2] = b.whole;
        out[3] = (n + 127) / 128;
    } else {
        const mm::PairPlan b = mm::pair_plan(s, sms);
        const int64_t columns = mode == kPlain ? b.width : 128;
        out[1] = b.split;
        out[2] = b.width;
        out[3] = (t + 255) / 256 * ((n + columns - 1) / columns);
    }
    out[4] = s.stages();
}
"""
_lib = None


def plan_of(kind, mode, t, n, k, f32=False, ldq=0):
    """A dict: few (tokens), split, tiles, stages of K, and width (pairs) or tokens and whole (few)."""
    global _lib
    if _lib is None:
        with tempfile.TemporaryDirectory() as d:
            src, so = os.path.join(d, "plan.cpp"), os.path.join(d, "plan.so")
            with open(src, "w") as f:
                f.write(SOURCE)
            subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2606_07618_gb300", "csrc"),
                            src, "-o", so], check=True)
            _lib = ctypes.CDLL(so)
        _lib.plan_of.argtypes = [ctypes.c_int] * 3 + [ctypes.c_int64] * 4 + [ctypes.c_int, ctypes.POINTER(ctypes.c_int64)]
    out = (ctypes.c_int64 * 5)()
    _lib.plan_of(kind, mode, int(f32), t, n, k, ldq, SMS, out)
    p = {"few": bool(out[0]), "split": out[1], "tiles": out[3], "stages": out[4]}
    if p["few"]:
        p.update(tokens=16 if t <= 16 else 32 if t <= 32 else 64, whole=bool(out[2]))
    else:
        p.update(width=out[2], walks=out[1] == 1 and out[3] > SMS // 2)      # whether a pair walks more than one tile
    return p


def up(n, to):
    return -(-n // to) * to


def matmul(fmt, m, n, k, f32=False):
    return plan_of(fmt, PLAIN, m, n, k, f32)


def matmul_grads(m, n, k, ldd=None):
    """dA and dB; ldd: dD's row stride."""
    ldd = ldd or n
    ldd = ldd if ldd % 8 == 0 else up(n, 8)
    return plan_of(BF16, PLAIN, m, k, n, ldq=ldd), plan_of(BF16, PLAIN, n, k, m, ldq=ldd)


def gated(fmt, t, f, d):
    return plan_of(fmt, GATED, t, f, d)


def gated_grads(fmt, t, f, d):
    """The recompute, d_x, and both weights' gradients; d_x's second part of K starts at stage `part` (NVFP4)."""
    fp = up(f, 128)
    x = plan_of(BF16, PLAIN, t, d, 2 * fp, ldq=2 * fp)
    x["part"] = fp // 64 if fmt == NV else 0
    return plan_of(fmt, GRAD, t, f, d), x, plan_of(BF16, PLAIN, fp + f, d, t, ldq=2 * fp)
