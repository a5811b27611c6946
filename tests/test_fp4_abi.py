"""include/nvfp4mm.h: every declared entry point is exported, and bad arguments are refused on the
host before any launch (no GPU needed; the pointers are never dereferenced)."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

import fp4_reference as R
from conftest import ROOT

FAKE = 0x10000000
OK, INVALID, UNSUPPORTED, ALIGNMENT, RANGE = 0, 1, 2, 3, 4


@pytest.fixture(scope="module")
def B():
    from paper_2606_07618_gb300 import binding
    binding.lib()
    return binding


def test_header_and_exports(B):
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "nvfp4mm.h")).read(), flags=re.S)
    names = re.findall(r"^(?:nvfp4_status|size_t)\s+([a-z0-9_]+)\s*\(", src, re.M)
    assert sorted(names) == sorted(["mxfp4_quantize", "mxfp4_dequantize", "fp4_matmul", "fp4_matmul_backward_workspace",
                                    "fp4_matmul_backward", "fp4_gated_ff", "fp4_gated_ff_backward_workspace",
                                    "fp4_gated_ff_backward", "fp4_selftest_wait_timeout"])
    for n in names:
        assert hasattr(B.lib(), n), n


def _op(B, codes=FAKE, sf=FAKE + 0x800000, S=None):
    return ctypes.byref(B.Fp4Operand(codes, sf, S))


def test_quantise_refusals(B):
    L = B.lib()
    q = lambda x=FAKE, dt=0, rows=4, cols=64, ld=64, codes=FAKE + 0x100000, lin=FAKE + 0x200000, swz=None, st=None: \
        L.mxfp4_quantize(x, dt, rows, cols, ld, codes, lin, swz, st, None)
    assert q(rows=0) == OK and q(cols=0, ld=0) == OK
    assert q(dt=2) == INVALID and q(rows=-1) == INVALID and q(cols=48) == INVALID
    assert q(x=None) == INVALID and q(codes=None) == INVALID and q(lin=None) == INVALID
    assert q(ld=63) == INVALID                                     # rows overlap
    assert q(x=FAKE + 1) == ALIGNMENT and q(dt=1, x=FAKE + 2) == ALIGNMENT
    assert q(codes=FAKE + 0x100004) == ALIGNMENT and q(swz=FAKE + 0x300002) == ALIGNMENT
    assert q(codes=FAKE) == INVALID and q(lin=FAKE + 0x100010) == INVALID   # overlaps
    assert q(rows=2 ** 40, ld=2 ** 40) == RANGE and q(cols=2 ** 31, ld=2 ** 31) == RANGE
    d = lambda codes=FAKE, sf=FAKE + 0x100000, lay=2, rows=4, cols=64, out=FAKE + 0x200000, dt=1: \
        L.mxfp4_dequantize(codes, sf, lay, rows, cols, out, dt, None)
    assert d(rows=0) == OK and d(lay=3) == INVALID and d(dt=9) == INVALID and d(cols=16) == INVALID
    assert d(codes=None) == INVALID and d(out=FAKE + 0x200008) == ALIGNMENT and d(out=FAKE) == INVALID


@pytest.mark.parametrize("rows,cols", [(17, 2 ** 30), (64, 2 ** 30), (2 ** 20, 2 ** 27 + 32)])
def test_conversions_refuse_what_their_counts_cannot_hold(B, rows, cols):
    """128 rows (or all) of more than 2^34 elements; at that size the call goes on to its other arguments."""
    L = B.lib()
    q = lambda r, c: L.mxfp4_quantize(FAKE, 0, r, c, c, None, None, None, None, None)
    d = lambda r, c: L.mxfp4_dequantize(None, FAKE, 2, r, c, FAKE, 0, None)
    assert q(rows, cols) == RANGE and d(rows, cols) == RANGE
    assert q(16, 2 ** 30) == INVALID and d(128, 2 ** 27) == INVALID and q(2 ** 20, 2 ** 27) == INVALID


def test_matmul_refusals(B):
    L = B.lib()
    mm = lambda fmt=0, a=None, b=None, m=4, n=8, k=64, D=FAKE + 0x2000000, dt=0, ld=8, st=None: \
        L.fp4_matmul(fmt, a or _op(B), b or _op(B, FAKE + 0x1000000, FAKE + 0x1800000), m, n, k, D, dt, ld, st, None)
    assert mm(m=0) == OK and mm(n=0) == OK
    assert mm(fmt=2) == INVALID and mm(dt=5) == INVALID and mm(m=-1) == INVALID
    assert mm(k=0) == UNSUPPORTED and mm(k=48) == UNSUPPORTED
    assert mm(D=None) == INVALID and mm(ld=7) == INVALID
    assert mm(a=_op(B, None)) == INVALID and mm(b=_op(B, FAKE, None)) == INVALID
    assert mm(fmt=1, a=_op(B, S=FAKE + 0x900000)) == INVALID       # MXFP4 has no global scale
    assert mm(a=_op(B, FAKE + 8)) == ALIGNMENT and mm(a=_op(B, FAKE, FAKE + 0x800004)) == ALIGNMENT
    assert mm(a=_op(B, S=FAKE + 0x900002)) == ALIGNMENT
    assert mm(D=FAKE + 0x2000001) == ALIGNMENT and mm(dt=1, D=FAKE + 0x2000002) == ALIGNMENT
    assert mm(D=FAKE) == INVALID                                   # over A's codes
    assert mm(m=2 ** 40) == RANGE and mm(k=2 ** 31) == RANGE and mm(n=2 ** 20, ld=2 ** 62) == RANGE
    assert L.fp4_selftest_wait_timeout(0, _op(B), _op(B, FAKE + 0x1000000, FAKE + 0x1800000), 4, 8, 64, FAKE + 0x2000000, 0, 8,
                                       None, None) == INVALID           # its status word is required
    w = L.fp4_matmul_backward_workspace(4, 8, 64)
    assert w > 0 and L.fp4_matmul_backward_workspace(0, 8, 64) == 0 and L.fp4_matmul_backward_workspace(-1, 8, 64) == 0
    bw = lambda dD=FAKE + 0x2000000, dA=FAKE + 0x2100000, dB=FAKE + 0x2200000, ws=FAKE + 0x3000000, wsb=w, ldd=8, lda=64: \
        L.fp4_matmul_backward(0, _op(B), _op(B, FAKE + 0x1000000, FAKE + 0x1800000), 4, 8, 64, dD, ldd, dA, lda, dB, 64,
                              None, ws, wsb, None)
    assert bw(dA=None, dB=None) == INVALID and bw(dD=None) == INVALID and bw(ws=None) == INVALID
    assert bw(wsb=w - 1) == INVALID and bw(ws=FAKE + 0x3000080) == ALIGNMENT and bw(ldd=7) == INVALID and bw(lda=63) == INVALID
    assert bw(dA=FAKE + 0x2000000) == INVALID and bw(ws=FAKE + 0x2000000) == INVALID


def test_gated_refusals(B):
    L = B.lib()
    x = lambda: _op(B)
    g = lambda: _op(B, FAKE + 0x1000000, FAKE + 0x1800000)
    u = lambda: _op(B, FAKE + 0x2000000, FAKE + 0x2800000)
    gf = lambda fmt=0, act=0, t=4, f=64, d=64, h=FAKE + 0x3000000, ld=64, hc=None, hs=None: \
        L.fp4_gated_ff(fmt, act, x(), g(), u(), t, f, d, h, ld, hc, hs, None, None)
    assert gf(t=0) == OK and gf(f=0) == OK
    assert gf(act=2) == INVALID and gf(fmt=-1) == INVALID and gf(d=16) == UNSUPPORTED and gf(t=-4) == INVALID
    assert gf(h=None) == INVALID and gf(hc=FAKE + 0x3100000) == INVALID and gf(hs=FAKE + 0x3100000) == INVALID
    assert gf(f=40, hc=FAKE + 0x3100000, hs=FAKE + 0x3200000) == INVALID   # not whole MXFP4 blocks
    assert gf(hc=FAKE + 0x3100008, hs=FAKE + 0x3200000) == ALIGNMENT and gf(ld=63) == INVALID
    assert gf(h=FAKE + 0x1000000) == INVALID
    w = L.fp4_gated_ff_backward_workspace(4, 64, 64)
    gb = lambda dh=FAKE + 0x3000000, dx=FAKE + 0x3100000, dg=FAKE + 0x3200000, du=FAKE + 0x3300000, h=None, wsb=w, act=0, ldw=64: \
        L.fp4_gated_ff_backward(0, act, x(), g(), u(), 4, 64, 64, dh, 64, dx, 64, dg, du, ldw, h, 64, None, FAKE + 0x4000000,
                                wsb, None)
    assert gb(dh=None) == INVALID and gb(dg=None) == INVALID and gb(dx=None, dg=None, du=None) == INVALID
    assert gb(wsb=w - 256) == INVALID and gb(act=3) == INVALID and gb(ldw=60) == INVALID
    assert gb(dx=FAKE + 0x3000000) == INVALID and gb(h=FAKE + 0x3100000) == INVALID


def test_gradients_without_rows_check_what_they_zero(B):
    """Zeros are written only where the output's own arguments hold; nothing to write is no error."""
    L = B.lib()
    mb = lambda m, n, dA, lda, dB, ldb: L.fp4_matmul_backward(0, None, None, m, n, 64, None, n, dA, lda, dB, ldb, None, None, 0, None)
    assert mb(0, 8, None, 64, None, 64) == OK and mb(8, 0, None, 64, None, 64) == OK and mb(0, 0, FAKE, 64, FAKE, 64) == OK
    assert mb(0, 8, None, 64, FAKE, 63) == INVALID and mb(0, 8, None, 64, FAKE + 1, 64) == ALIGNMENT
    assert mb(8, 0, FAKE, 63, None, 64) == INVALID
    gb = lambda t, f, dx, dg, du, ldw: L.fp4_gated_ff_backward(0, 0, None, None, None, t, f, 64, None, f, dx, 64, dg, du, ldw,
                                                                 None, f, None, None, 0, None)
    assert gb(0, 8, None, None, None, 64) == OK and gb(8, 0, None, None, None, 64) == OK
    assert gb(0, 8, None, FAKE, None, 64) == INVALID and gb(0, 8, None, FAKE, FAKE + 64, 64) == INVALID     # overlap
    assert gb(0, 8, None, FAKE, FAKE + 0x10000, 60) == INVALID and gb(8, 0, FAKE + 1, None, None, 64) == ALIGNMENT


def test_gated_without_rows_takes_null_outputs(B):
    gf = lambda t, f, hc=None, hs=None: B.lib().fp4_gated_ff(0, 0, None, None, None, t, f, 64, None, f, hc, hs, None, None)
    assert gf(0, 64) == OK and gf(4, 0) == OK and gf(0, 64, FAKE, None) == INVALID


def test_binding_refuses_shapes_and_types(B):
    z = lambda *s, dt=torch.uint8: torch.zeros(*s, dtype=dt)
    op = lambda rows, cols: (z(rows, cols // 2), z(B.swizzled_bytes(rows, cols)), None)
    with pytest.raises(ValueError):
        B.fp4_matmul(0, op(4, 64), op(4, 96), z(4, 4, dt=torch.float32))
    with pytest.raises(ValueError):
        B.fp4_matmul(0, op(4, 64), op(4, 64), z(4, 5, dt=torch.float32))
    with pytest.raises(ValueError):
        B.fp4_matmul(0, (z(4, 32), z(16), None), op(4, 64), z(4, 4, dt=torch.float32))       # scales too short
    with pytest.raises(ValueError):
        B.fp4_matmul(0, op(4, 64), op(4, 64), z(4, 4, dt=torch.float32).t())
    with pytest.raises(TypeError):
        B.fp4_matmul(0, op(4, 64), op(4, 64), z(4, 4, dt=torch.float16))
    with pytest.raises(TypeError):
        B.fp4_gated_ff(0, 0, op(4, 64), op(8, 64), op(8, 64), z(4, 8, dt=torch.float32))
    with pytest.raises(ValueError):
        B.fp4_gated_ff(0, 0, op(4, 64), op(8, 64), op(9, 64), z(4, 8, dt=torch.bfloat16))
    with pytest.raises(ValueError):
        B.mxfp4_quantize(z(64, 4, dt=torch.float32).t(), z(4, 32), z(4, 2))


def test_binding_refuses_buffers_that_are_too_small(B):
    """Buffers that a kernel would run past: short ones, and views whose elements are not in a row."""
    z = lambda *s, dt=torch.uint8: torch.zeros(*s, dtype=dt)
    x, codes, lin, swz = z(4, 64, dt=torch.float32), z(4, 32), z(4, 2), z(B.mx_swizzled_bytes(4, 64))
    for bad in ((codes[:3], lin, None), (codes, lin[:3], None), (codes, None, swz[:-1]), (z(4, 64)[:, ::2], lin, None),
                (codes, None, z(1).expand(swz.numel()))):
        with pytest.raises(ValueError):
            B.mxfp4_quantize(x, *bad)
    for bad in ((codes[:3], lin, 1), (codes, lin[:3], 1), (codes, lin, 2)):
        with pytest.raises(ValueError):
            B.mxfp4_dequantize(*bad, 4, 64, x)
    with pytest.raises(ValueError):
        B.mxfp4_dequantize(codes, lin, 1, 4, 64, x[:3])
    op = lambda rows, cols: (z(rows, cols // 2), z(B.swizzled_bytes(rows, cols)), None)
    with pytest.raises(ValueError):
        B.fp4_matmul(0, (z(4, 32), z(1).expand(512), None), op(4, 64), z(4, 4, dt=torch.float32))
    with pytest.raises(ValueError):
        B.fp4_gated_ff(0, 0, op(4, 64), op(32, 64), op(32, 64), None, z(4, 16), z(1).expand(512))
    with pytest.raises(ValueError):
        B.fp4_matmul_backward(0, op(4, 64), op(8, 64), z(4, 8, dt=torch.bfloat16), z(4, 64, dt=torch.bfloat16), None,
                              z(1).expand(2 ** 20))


# ------------------------------------------------------------------ the reference itself
def test_reference_rounds_as_the_definition():
    x = np.zeros((1, 32))
    x[0, :9] = [4, 5, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, -0.3]
    codes, sf = R.mxfp4(x)
    assert sf[0, 0] == 127
    assert R.values(codes, sf, R.MX)[0, :9].tolist() == [4, 4, 0, 1, 1, 2, 2, 4, -0.5]
    x[0, 0] = 7.9                                                  # past 6: to 6, the scale stays
    codes, sf = R.mxfp4(x)
    assert sf[0, 0] == 127 and R.values(codes, sf, R.MX)[0, 0] == 6


def test_reference_decodes_as_torch():
    sf = np.arange(127, dtype=np.uint8)
    assert np.array_equal(R.scale_values(sf, R.NV), torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy())


@pytest.mark.parametrize("act", [0, 1])
def test_reference_gradients_are_the_differences(act):
    g = np.random.default_rng(1)
    x, wg, wu, dh = g.standard_normal((5, 8)), g.standard_normal((7, 8)), g.standard_normal((7, 8)), g.standard_normal((5, 7))
    grads = R.gated_grad(act, x, wg, wu, dh)
    for i in range(3):
        at = [x, wg, wu]
        v = g.standard_normal(at[i].shape)
        at_plus, at_minus = list(at), list(at)
        at_plus[i], at_minus[i] = at[i] + 1e-5 * v, at[i] - 1e-5 * v
        diff = ((dh * R.gated(act, *at_plus)).sum() - (dh * R.gated(act, *at_minus)).sum()) / 2e-5
        assert abs((grads[i] * v).sum() - diff) <= 1e-6 * (1 + abs(diff))
