"""The kernels' paths that sizes lead to: each ring and split of the few-token kernel, tiles of every width, pairs of
CTAs that walk more tiles than one, K split over a cluster, and d_x's two parts of K under each of them.  Each against
64 bits, within the bounds that test_gpu_fp4.py derives.  The path beside a shape is what csrc/fp4_plan.h chooses for it
on 152 SMs, which test_fp4_plans.py checks without a GPU: (tokens, split, whole SM's ring) of few tokens, or (width,
split, whether a pair walks several tiles)."""
import numpy as np
import pytest
import torch

import fp4_reference as R
from test_gpu_fp4 import (DEV, B, H, U, Held, bf16, gated_bounds, gated_operands, grad_bounds, guarded, near,  # noqa: F401
                          quantised, sum_bound)

pytestmark = pytest.mark.gpu

MATMUL = [((9, 300, 800), (16, 4, False)), ((3, 9800, 64), (16, 1, True)), ((20, 9800, 160), (32, 1, True)),
          ((20, 19500, 64), (32, 1, False)), ((25, 200, 288), (32, 2, False)), ((31, 300, 1056), (32, 4, False)),
          ((40, 19500, 96), (64, 1, False)), ((50, 9900, 288), (64, 1, True)), ((64, 5900, 8192), (64, 4, False)), ((37, 200, 8224), (64, 8, False)),
          ((1700, 2561, 64), (128, 1, True)), ((100, 3900, 16384), (128, 2, False)), ((1300, 1111, 16384), (256, 2, False)),
          ((1300, 3300, 608), (256, 1, True))]

GATED = [((9, 320, 800), (16, 4, False)), ((3, 9824, 64), (16, 1, True)), ((20, 9824, 160), (32, 1, True)),
         ((20, 19488, 64), (32, 1, False)), ((25, 192, 288), (32, 2, False)), ((31, 320, 1056), (32, 4, False)),
         ((32, 96, 2080), (32, 8, False)), ((40, 19488, 96), (64, 1, False)), ((50, 9920, 288), (64, 1, True)),
         ((64, 5920, 8192), (64, 4, False)), ((37, 192, 8224), (64, 8, False)), ((1300, 2080, 96), (256, 1, True)), ((1300, 2112, 352), (256, 1, True)),
         ((1300, 2049, 352), (256, 1, True)), ((700, 4000, 608), (256, 1, True)), ((300, 2080, 12320), (256, 2, False))]

MATMUL_GRADS = [((64, 4096, 256), (128, 4, False), (128, 1, False)), ((77, 4096, 4096), (128, 2, False), (256, 1, True)),
                ((1024, 4096, 4096), (224, 1, False), (224, 1, True)), ((555, 249, 3296), (224, 1, False), (128, 1, False)),
                ((600, 250, 7200), (224, 1, True), (128, 1, False)), ((64, 2200, 1952), (256, 4, False), (256, 1, False)),
                ((2700, 40, 1568), (128, 1, True), (128, 4, False)), ((40, 2700, 1568), (128, 4, False), (128, 1, True)),
                ((200, 320, 5472), (128, 1, False), (224, 1, False)), ((5000, 300, 2560), (256, 1, True), (256, 2, False)),
                ((4100, 1000, 1088), (256, 1, True), (128, 2, False))]

GATED_GRADS = [((64, 2000, 256), (256, 1, False), (128, 4, False), (128, 1, False)),
               ((64, 2000, 3968), (256, 1, False), (128, 2, False), (256, 1, True)),
               ((70, 2081, 4736), (256, 1, False), (256, 2, False), (256, 1, True)),
               ((2100, 1300, 256), (256, 1, True), (256, 4, False), (128, 1, False)),
               ((1300, 2049, 352), (256, 1, True), (256, 4, False), (128, 1, False)),
               ((2700, 70, 1568), (256, 1, False), (128, 1, True), (128, 4, False)),
               ((522, 100, 6816), (256, 1, False), (224, 1, True), (128, 1, False)),
               ((773, 50, 8608), (256, 4, False), (256, 1, True), (128, 1, False)),
               ((216, 9878, 160), (256, 1, True), (128, 4, False), (224, 1, True)),
               ((4100, 130, 1120), (256, 1, False), (224, 1, True), (256, 4, False)),
               ((300, 1100, 8224), (256, 2, False), (224, 1, False), (256, 1, True)),
               ((261, 60, 8736), (256, 4, False), (256, 1, False), (128, 1, False))]


@pytest.mark.parametrize("fmt", [R.NV, R.MX])
@pytest.mark.parametrize("shape,path", MATMUL)
def test_matmul(B, fmt, shape, path):
    m, n, k = shape
    a, b = Held(m, k, fmt, m + n), Held(n, k, fmt, n + k)
    want, bound = a.v @ b.v.T, sum_bound(a.v, b.v, k)
    for out in (torch.float32, torch.bfloat16):
        D, check = guarded(m, n, out, n + 3, 1)
        B.fp4_matmul(fmt, a.op, b.op, D)
        near(D, want, bound + (H * np.abs(want) if out == torch.bfloat16 else 0))
        check()
        whole = torch.empty(m, n, dtype=out, device=DEV)
        B.fp4_matmul(fmt, a.op, b.op, whole)
        assert torch.equal(whole, D)


@pytest.mark.parametrize("fmt", [R.NV, R.MX])
@pytest.mark.parametrize("act", [0, 1])
@pytest.mark.parametrize("shape,path", GATED)
def test_gated(B, fmt, act, shape, path):
    t, f, d = shape
    x, wg, wu = gated_operands(t, f, d, fmt)
    want, bound, *_ = gated_bounds(act, x.v, wg.v, wu.v, d)
    bound = bound + H * (np.abs(want) + bound) + 2.0 ** -133
    h, check = guarded(t, f, torch.bfloat16)
    if f % 32:
        B.fp4_gated_ff(fmt, act, x.op, wg.op, wu.op, h)
    else:
        codes = torch.full((t, f // 2), 0xAA, dtype=torch.uint8, device=DEV)
        sf = torch.full((B.mx_swizzled_bytes(t, f),), 0xAA, dtype=torch.uint8, device=DEV)
        B.fp4_gated_ff(fmt, act, x.op, wg.op, wu.op, h, codes, sf)
        qc, _, qs, _ = quantised(B, h)
        assert torch.equal(codes, qc) and torch.equal(sf, qs)
    near(h, want, bound)
    check()


@pytest.mark.parametrize("fmt", [R.NV, R.MX])
@pytest.mark.parametrize("shape,pa,pb", MATMUL_GRADS)
def test_matmul_grads(B, fmt, shape, pa, pb):
    m, n, k = shape
    a, b = Held(m, k, fmt, 11), Held(n, k, fmt, 12)
    dD = bf16(np.random.default_rng(13).standard_normal((m, n)))
    d = dD.double().numpy()
    ws = torch.empty(B.fp4_matmul_backward_workspace(m, n, k), dtype=torch.uint8, device=DEV)
    (dA, ca), (dB, cb) = guarded(m, k, torch.bfloat16), guarded(n, k, torch.bfloat16)
    B.fp4_matmul_backward(fmt, a.op, b.op, dD.to(DEV), dA, dB, ws)
    wa, wb = d @ b.v, d.T @ a.v
    near(dA, wa, (n + 4) * U * (np.abs(d) @ np.abs(b.v)) + H * np.abs(wa), "dA")
    near(dB, wb, (m + 4) * U * (np.abs(d).T @ np.abs(a.v)) + H * np.abs(wb), "dB")
    ca(), cb()


@pytest.mark.parametrize("fmt", [R.NV, R.MX])
@pytest.mark.parametrize("shape,pr,px,pw", GATED_GRADS)
def test_gated_grads(B, fmt, shape, pr, px, pw):
    t, f, d = shape
    x, wg, wu = gated_operands(t, f, d, fmt)
    dh = bf16(np.random.default_rng(4).standard_normal((t, f)))
    ws = torch.empty(B.fp4_gated_ff_backward_workspace(t, f, d), dtype=torch.uint8, device=DEV)
    out = [guarded(r, c, torch.bfloat16) for r, c in ((t, d), (f, d), (f, d), (t, f))]
    B.fp4_gated_ff_backward(fmt, 0, x.op, wg.op, wu.op, dh.to(DEV), *(o[0] for o in out), ws)
    for (got, check), (want, bound), what in zip(out, grad_bounds(0, x.v, wg.v, wu.v, dh.double().numpy(), d),
                                                 ("dx", "dgate", "dup")):
        near(got, want, bound, what)
        check()
    want, bound, *_ = gated_bounds(0, x.v, wg.v, wu.v, d)
    near(out[3][0], want, bound + H * (np.abs(want) + bound) + 2.0 ** -133, "h")
    out[3][1]()


# few tokens alone and split, pairs alone, walking and split
@pytest.mark.parametrize("t,f,d", [(3, 96, 64), (20, 192, 800), (64, 96, 8224), (100, 224, 288), (1300, 2080, 96), (70, 192, 8224)])
def test_gated_results_that_are_not_finite(B, t, f, d):
    """Rows of x large enough that h overflows: blocks with an infinity become scale code 0 and signs, reported in the
    status word; the blocks of the other rows are those of a call without such rows."""
    x, wg, wu = gated_operands(t, f, d, R.MX)
    outs = []
    for grown in (False, True):
        sf = x.sf.copy()
        if grown:
            sf[1::7] += 80                                       # g and u of about 2^80: their product passes 2^128
        op = (x.op[0], torch.from_numpy(R.swizzle(sf)).to(DEV), None)
        h = torch.empty(t, f, dtype=torch.bfloat16, device=DEV)
        codes = torch.full((t, f // 2), 0xAA, dtype=torch.uint8, device=DEV)
        hs = torch.full((B.mx_swizzled_bytes(t, f),), 0xAA, dtype=torch.uint8, device=DEV)
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        B.fp4_gated_ff(R.MX, 0, op, wg.op, wu.op, h, codes, hs, status)
        qc, lin, qs, st = quantised(B, h)
        assert torch.equal(codes, qc) and torch.equal(hs, qs) and status.item() == st == int(grown)
        outs.append((h, codes, lin))
    (h0, c0, _), (h1, c1, lin) = outs
    rows = torch.zeros(t, dtype=torch.bool, device=DEV)
    rows[1::7] = True
    bad = ~torch.isfinite(h1).view(t, -1, 32).all(-1)
    assert bool(bad[rows].any(1).all()) and not bool(bad[~rows].any())
    assert torch.equal(h0[~rows], h1[~rows]) and torch.equal(c0[~rows], c1[~rows])
    assert not bool(lin[bad].any()) and not bool((c1.view(t, -1, 16)[bad] & 0x77).any())


# the few-token kernel forward, pairs in the gradients' call: sums in another order
@pytest.mark.parametrize("fmt", [R.NV, R.MX])
@pytest.mark.parametrize("t,f,d", [(1, 200, 4096), (32, 320, 4128), (50, 96, 8224)])
def test_the_gradients_h_of_few_tokens(B, fmt, t, f, d):
    """The forward result that the gradients' call writes, within the bound of either's sums."""
    x, wg, wu = gated_operands(t, f, d, fmt)
    ws = torch.empty(B.fp4_gated_ff_backward_workspace(t, f, d), dtype=torch.uint8, device=DEV)
    h, fwd = (torch.empty(t, f, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    dx = torch.empty(t, d, dtype=torch.bfloat16, device=DEV)
    dh = bf16(np.random.default_rng(4).standard_normal((t, f))).to(DEV)
    B.fp4_gated_ff_backward(fmt, 0, x.op, wg.op, wu.op, dh, dx, None, None, h, ws)
    B.fp4_gated_ff(fmt, 0, x.op, wg.op, wu.op, fwd)
    want, bound, *_ = gated_bounds(0, x.v, wg.v, wu.v, d)
    for got in (h, fwd):
        near(got, want, bound + H * (np.abs(want) + bound) + 2.0 ** -133)
