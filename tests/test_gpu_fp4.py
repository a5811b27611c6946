"""MXFP4 quantisation, products of 4-bit matrices, the gated feed-forward and their gradients
against 64-bit references, at sizes and values where they can go wrong.

Bounds.  U = 2^-23 bounds one fp32 addition that truncates, H = 2^-8 one rounding to bf16 (8 significant bits).
A product's sums are of exact terms; it makes at most one addition a term, so its error is
within (K + 4) U sum|a b| (the scales' products included), plus H |result| for bf16 outputs.
The gated form's and the gradients' bounds follow from those of g and u, with |act'| < 1.13,
|act''| < 1.2 and 2^-18 for the activation's own error (exp and a quotient of a few ulps,
and what its argument's rounding makes of |g| < 2^4), and one H for each rounding to bf16."""
import numpy as np
import pytest
import torch

import fp4_reference as R

pytestmark = pytest.mark.gpu
DEV = "cuda"
U, H = 2.0 ** -23, 2.0 ** -8


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2606_07618_gb300 import binding
    binding.lib()
    return binding


class Held:
    """A random quantised matrix on the GPU and its values in 64 bits."""

    def __init__(self, rows, cols, fmt, seed, spread=3):
        self.codes, self.sf, self.S = R.random_matrix(rows, cols, fmt, seed, spread)
        self.v = R.values(self.codes, self.sf, fmt, 1.0 if self.S is None else self.S)
        S = None if self.S is None else torch.tensor([self.S], device=DEV)
        self.op = (torch.from_numpy(self.codes).to(DEV), torch.from_numpy(R.swizzle(self.sf)).to(DEV), S)


def bf16(a):
    return torch.from_numpy(np.asarray(a, np.float32)).to(torch.bfloat16)


def host(t):
    return t.double().cpu().numpy()


def guarded(rows, cols, dtype, ld=None, shift=0):
    """A [rows, cols] output inside a buffer of a known value; check() says that nothing else was written."""
    ld = ld or cols
    buf = torch.full((rows * ld + shift + 64,), 7.0, dtype=dtype, device=DEV)
    out = buf[shift:shift + rows * ld].view(rows, ld)[:, :cols]

    def check():
        m = torch.ones_like(buf, dtype=torch.bool)
        m[shift:shift + rows * ld].view(rows, ld)[:, :cols] = False
        assert bool((buf[m] == 7.0).all()), "written outside the output"
    return out, check


def near(got, want, bound, what=""):
    got, bound = host(got), np.broadcast_to(bound, want.shape)
    assert got.shape == want.shape
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), (what, int(bad.sum()), got[bad][:4], want[bad][:4], bound[bad][:4])


# ------------------------------------------------------------------ quantisation
def quantised(B, x, linear=True, swizzled=True):
    rows, cols = x.shape
    codes = torch.full((rows, cols // 2), 0xAA, dtype=torch.uint8, device=DEV)
    lin = torch.full((rows, cols // 32), 0xAA, dtype=torch.uint8, device=DEV) if linear else None
    swz = torch.full((B.mx_swizzled_bytes(rows, cols),), 0xAA, dtype=torch.uint8, device=DEV) if swizzled else None
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    B.mxfp4_quantize(x, codes, lin, swz, status)
    torch.cuda.synchronize()
    return codes, lin, swz, status.item()


def check_quantised(B, x, **kw):
    want_codes, want_sf = R.mxfp4(host(x))
    codes, lin, swz, status = quantised(B, x, **kw)
    assert np.array_equal(codes.cpu().numpy(), want_codes)
    if lin is not None:
        assert np.array_equal(lin.cpu().numpy(), want_sf)
    if swz is not None:
        assert np.array_equal(swz.cpu().numpy(), R.swizzle(want_sf))
    return want_codes, want_sf, status


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols", [(1, 32), (1, 96), (3, 64), (127, 160), (128, 128), (129, 416), (5, 4096), (700, 1056)])
def test_quantise_bit_exact(B, dtype, rows, cols):
    g = torch.Generator().manual_seed(rows * cols)
    x = (torch.randn(rows, cols, generator=g) * torch.exp(2 * torch.randn(rows, 1, generator=g))).to(dtype).to(DEV)
    assert check_quantised(B, x)[2] == 0
    check_quantised(B, x, linear=False)
    check_quantised(B, x, swizzled=False)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_quantise_ties_and_edges(B, dtype):
    """Every midpoint and its neighbours at several scales, the largest mantissa, signed zeros, subnormals."""
    mids = np.array([0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 6, 7, 7.96875, 4, 0.5, 1, 2, 3])
    rows = []
    for e in (-140, -133, -127, -126, -100, -3, 0, 5, 100, 125):
        with np.errstate(over="ignore"):
            block = np.concatenate([mids, -mids]) * np.ldexp(1.0, e)
        for eps in (0, 2.0 ** -7, -2.0 ** -7):
            r = block * (1 + eps)
            r[0], r[16] = 4 * np.ldexp(1.0, e), -0.0     # the block's maximum stays in its octave
            rows.append(np.where(np.abs(r) < 8 * np.ldexp(1.0, e), r, 7.5 * np.ldexp(1.0, e)))
    x = torch.tensor(np.array(rows), dtype=torch.float64).to(torch.float32).to(dtype)
    x = x[torch.isfinite(x).all(1)].to(DEV)
    check_quantised(B, x)
    z = torch.zeros(2, 64, dtype=dtype, device=DEV)
    z[1, ::2] = -0.0
    check_quantised(B, z)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
def test_quantise_nonfinite_block_is_zero_and_flagged(B, dtype, value):
    x = torch.randn(5, 96, generator=torch.Generator().manual_seed(3)).to(dtype).to(DEV)
    x[2, 40] = value
    codes, lin, _, status = quantised(B, x)
    assert status == 1
    assert lin[2, 1].item() == 0
    want = np.where(np.signbit(x[2, 32:64].float().cpu().numpy()), 8, 0)
    got = codes[2, 16:32].cpu().numpy()
    n = np.stack([got & 15, got >> 4], 1).reshape(-1)
    keep = np.arange(32) != 8 if value != value else np.ones(32, bool)   # a NaN's sign is free
    assert np.array_equal(n[keep], want[keep]) and (n & 7).max() == 0
    x[2, 32:64] = 0
    c2, l2 = R.mxfp4(host(x))
    codes[2, 16:32] = torch.from_numpy(c2[2, 16:32]).to(DEV)
    assert np.array_equal(codes.cpu().numpy(), c2) and np.array_equal(lin.cpu().numpy(), l2)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("offset,stride", [(0, 256), (8, 264), (4, 260), (1, 257), (16, 240)])
def test_quantise_strided(B, dtype, offset, stride):
    buf = torch.randn(33 * stride + 64, generator=torch.Generator().manual_seed(offset)).to(dtype).to(DEV)
    x = buf[offset:offset + 33 * stride].view(33, stride)[:, :192]
    check_quantised(B, x)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols", [(1, 32), (130, 416), (64, 2048)])
def test_dequantise_bit_exact(B, dtype, rows, cols):
    g = np.random.default_rng(rows)
    codes = g.integers(0, 256, (rows, cols // 2)).astype(np.uint8)
    sf = g.integers(0, 253, (rows, cols // 32)).astype(np.uint8)
    sf[0, 0] = 0
    want = torch.from_numpy(R.values(codes, sf, R.MX)).to(torch.float32).to(dtype)
    c = torch.from_numpy(codes).to(DEV)
    for layout, s in ((B.NVFP4_SF_LINEAR, sf), (B.NVFP4_SF_SWIZZLED, R.swizzle(sf))):
        out = torch.full((rows, cols), 7.0, dtype=dtype, device=DEV)
        B.mxfp4_dequantize(c, torch.from_numpy(np.ascontiguousarray(s)).to(DEV), layout, rows, cols, out)
        assert torch.equal(out.cpu(), want)


# ------------------------------------------------------------------ products
SHAPES = [(1, 1, 32), (1, 128, 256), (7, 129, 96), (16, 300, 320), (17, 128, 2080), (33, 1, 64), (64, 257, 512),
          (65, 96, 288), (128, 128, 256), (129, 130, 1024), (200, 384, 544), (300, 700, 1312)]


def sum_bound(a, b, k):
    return (k + 4) * U * (np.abs(a) @ np.abs(b).T)


@pytest.mark.parametrize("fmt", [R.NV, R.MX])
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_matmul(B, fmt, out, m, n, k):
    a, b = Held(m, k, fmt, m + n + k), Held(n, k, fmt, m * n + k)
    D, check = guarded(m, n, out)
    B.fp4_matmul(fmt, a.op, b.op, D)
    want = a.v @ b.v.T
    near(D, want, sum_bound(a.v, b.v, k) + (H * np.abs(want) if out == torch.bfloat16 else 0))
    check()


@pytest.mark.parametrize("fmt", [R.NV, R.MX])
@pytest.mark.parametrize("m,n,k", [(512, 512, 512), (257, 1000, 1056), (1025, 2049, 288), (1, 4096, 4096), (1030, 4100, 4128)])
def test_matmul_large(B, fmt, m, n, k):
    a, b = Held(m, k, fmt, 5), Held(n, k, fmt, 6)
    D, check = guarded(m, n, torch.float32)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    B.fp4_matmul(fmt, a.op, b.op, D, st)
    near(D, a.v @ b.v.T, sum_bound(a.v, b.v, k))
    assert st.item() == 0
    check()


@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("ld,shift", [(140, 0), (129, 0), (136, 1), (133, 3)])
@pytest.mark.parametrize("m", [5, 200, 600])
def test_matmul_strided_output(B, out, ld, shift, m):
    n, k = 129, 160
    a, b = Held(m, k, R.MX, 1), Held(n, k, R.MX, 2)
    D, check = guarded(m, n, out, ld, shift)
    B.fp4_matmul(R.MX, a.op, b.op, D)
    want = a.v @ b.v.T
    near(D, want, sum_bound(a.v, b.v, k) + (H * np.abs(want) if out == torch.bfloat16 else 0))
    check()


def test_matmul_scales_of_every_code(B):
    """Each finite E4M3 and a wide range of E8M0 codes as a scale, with S far from 1."""
    for fmt, sf in ((R.NV, np.arange(127, dtype=np.uint8)), (R.MX, np.arange(60, 187, dtype=np.uint8))):
        bl = R.block_of(fmt)
        codes = np.full((127, bl), 0x22, np.uint8)               # 1.0 everywhere, two blocks
        sfm = np.stack([sf, np.zeros_like(sf)], 1)
        codes[:, bl // 2:] = 0
        ones = np.full((3, bl), 0x22, np.uint8)
        one = np.full((3, 2), 127 if fmt == R.MX else 56, np.uint8)
        S = None if fmt == R.MX else torch.tensor([2.0 ** -20], device=DEV)
        k = 2 * bl
        op = lambda c, s: (torch.from_numpy(c).to(DEV), torch.from_numpy(R.swizzle(s)).to(DEV), S)  # noqa: E731
        D = torch.empty(3, 127, device=DEV)
        B.fp4_matmul(fmt, op(ones, one), op(codes, sfm), D)
        want = bl * R.scale_values(sf, fmt) * (1.0 if S is None else 2.0 ** -40)
        assert k % 32 == 0 and np.array_equal(host(D), np.tile(want, (3, 1)))


def test_matmul_zero_and_nan_scales(B):
    """A zero scale gives zeros; a NaN scale code reaches its own row and no other."""
    a, b = Held(40, 96, R.MX, 1), Held(50, 96, R.MX, 2)
    a.sf[3], a.sf[7, 1] = 0, 255
    a.codes[3] = 0
    D = torch.empty(40, 50, device=DEV)
    B.fp4_matmul(R.MX, (torch.from_numpy(a.codes).to(DEV), torch.from_numpy(R.swizzle(a.sf)).to(DEV), None), b.op, D)
    got = host(D)
    assert (got[3] == 0).all() and np.isnan(got[7]).all() and np.isfinite(np.delete(got, 7, 0)).all()


@pytest.mark.parametrize("fmt", [R.NV, R.MX])
@pytest.mark.parametrize("m,n,k", [(1, 1, 32), (5, 37, 96), (64, 128, 256), (130, 257, 416), (300, 520, 672)])
def test_matmul_backward(B, fmt, m, n, k):
    a, b = Held(m, k, fmt, 11), Held(n, k, fmt, 12)
    dD = bf16(np.random.default_rng(13).standard_normal((m, n)))
    d = dD.double().numpy()
    ws = torch.empty(B.fp4_matmul_backward_workspace(m, n, k), dtype=torch.uint8, device=DEV)
    dA, ca = guarded(m, k, torch.bfloat16)
    dB, cb = guarded(n, k, torch.bfloat16)
    B.fp4_matmul_backward(fmt, a.op, b.op, dD.to(DEV), dA, dB, ws)
    wa, wb = d @ b.v, d.T @ a.v
    near(dA, wa, (n + 4) * U * (np.abs(d) @ np.abs(b.v)) + H * np.abs(wa), "dA")
    near(dB, wb, (m + 4) * U * (np.abs(d).T @ np.abs(a.v)) + H * np.abs(wb), "dB")
    ca(), cb()
    one, c1 = guarded(m, k, torch.bfloat16, k + 3, 1)
    B.fp4_matmul_backward(fmt, a.op, b.op, dD.to(DEV), one, None, ws)
    assert torch.equal(one, dA)
    c1()
    two = torch.empty_like(dB)
    wide = torch.zeros(m, n + 5, dtype=torch.bfloat16, device=DEV)
    wide[:, 2:2 + n] = dD.to(DEV)
    B.fp4_matmul_backward(fmt, a.op, b.op, wide[:, 2:2 + n], None, two, ws)
    assert torch.equal(two, dB)


# ------------------------------------------------------------------ gated feed-forward
def gated_bounds(act, x, wg, wu, k):
    """h, its bound without the last rounding, and g, u, their bounds."""
    g, u = x @ wg.T, x @ wu.T
    eg, eu = sum_bound(x, wg, k), sum_bound(x, wu, k)
    a, _ = R.act(act, g)
    ea = 1.13 * eg + 2.0 ** -18 * np.abs(a)
    return a * u, ea * (np.abs(u) + eu) + np.abs(a) * eu, g, u, eg, eu


def gated_operands(t, f, d, fmt, spread=1):
    x, wg, wu = Held(t, d, fmt, t + 1, spread), Held(f, d, fmt, f + 2, spread), Held(f, d, fmt, d + 3, spread)
    if fmt == R.MX:                                              # values of a layer's size: |g| of a few units
        for m, by in ((x, 1), (wg, 4 + int(np.log2(d)) // 2), (wu, 4 + int(np.log2(d)) // 2)):
            m.sf = (m.sf - by).astype(np.uint8)
            m.v = m.v * 2.0 ** -by
            m.op = (m.op[0], torch.from_numpy(R.swizzle(m.sf)).to(DEV), None)
    return x, wg, wu


@pytest.mark.parametrize("fmt", [R.NV, R.MX])
@pytest.mark.parametrize("act", [0, 1])
@pytest.mark.parametrize("t,f,d", [(1, 1, 32), (1, 200, 512), (13, 129, 96), (32, 128, 1056), (50, 320, 256), (77, 64, 288),
                                   (128, 384, 512), (333, 417, 544), (520, 1000, 288)])
def test_gated(B, fmt, act, t, f, d):
    x, wg, wu = gated_operands(t, f, d, fmt)
    h, check = guarded(t, f, torch.bfloat16)
    B.fp4_gated_ff(fmt, act, x.op, wg.op, wu.op, h)
    want, bound, *_ = gated_bounds(act, x.v, wg.v, wu.v, d)
    near(h, want, bound + H * (np.abs(want) + bound) + 2.0 ** -133)
    check()


def test_gated_far_from_zero(B):
    """Gates of +-2^12: SiLU and GELU are g and 0 there, and nothing overflows."""
    x, wg, wu = Held(3, 64, R.MX, 1), Held(40, 64, R.MX, 2, 0), Held(40, 64, R.MX, 3, 0)
    x.op[0][:] = 0x77                                            # 6 in every place
    wg.op[0][:20], wg.op[0][20:] = 0x77, 0xFF                    # +6, -6
    for act in (0, 1):
        h = torch.empty(3, 40, dtype=torch.bfloat16, device=DEV)
        B.fp4_gated_ff(R.MX, act, x.op, wg.op, wu.op, h)
        got = host(h)
        v = lambda m: R.values(m.op[0].cpu().numpy(), m.sf, R.MX)  # noqa: E731
        g, u = v(x) @ v(wg).T, v(x) @ v(wu).T
        assert (np.abs(g) > 100).all()
        want = np.where(g > 0, g, 0) * u
        assert (np.abs(got - want) <= 2 * H * np.abs(want) + (np.abs(u) * np.abs(g) * 1e-30)).all()


@pytest.mark.parametrize("fmt", [R.NV, R.MX])
@pytest.mark.parametrize("t,f,d", [(1, 32, 64), (5, 160, 256), (16, 1056, 512), (40, 128, 96), (100, 224, 288), (130, 416, 544),
                                   (520, 1024, 256)])
def test_gated_in_mxfp4_is_the_quantised_bf16_result(B, fmt, t, f, d):
    x, wg, wu = gated_operands(t, f, d, fmt)
    h = torch.empty(t, f, dtype=torch.bfloat16, device=DEV)
    codes = torch.full((t, f // 2), 0xAA, dtype=torch.uint8, device=DEV)
    sf = torch.full((B.mx_swizzled_bytes(t, f),), 0xAA, dtype=torch.uint8, device=DEV)
    B.fp4_gated_ff(fmt, 0, x.op, wg.op, wu.op, h, codes, sf)
    qc, _, qs, _ = quantised(B, h)
    assert torch.equal(codes, qc) and torch.equal(sf, qs)
    only, sf2 = torch.empty_like(codes), torch.empty_like(sf)
    B.fp4_gated_ff(fmt, 0, x.op, wg.op, wu.op, None, only, sf2)
    assert torch.equal(codes, only) and torch.equal(sf, sf2)


def grad_bounds(act, x, wg, wu, dh, k):
    h, _, g, u, eg, eu = gated_bounds(act, x, wg, wu, k)
    a, da = R.act(act, g)
    ea = 1.13 * eg + 2.0 ** -18 * np.abs(a)
    eda = 1.2 * eg + 2.0 ** -18
    dg, du = dh * u * da, dh * a
    # each rounded once to bf16, after a product with S for d_x
    edg = np.abs(dh) * (np.abs(u) * eda + eu * (np.abs(da) + eda))
    edu = np.abs(dh) * ea
    edg, edu = edg + (H + 2 * U) * (np.abs(dg) + edg), edu + (H + 2 * U) * (np.abs(du) + edu)
    t, f = dh.shape
    dx, dwg, dwu = dg @ wg + du @ wu, dg.T @ x, du.T @ x
    G, V = np.abs(dg) + edg, np.abs(du) + edu
    bx = edg @ np.abs(wg) + edu @ np.abs(wu) + (2 * f + 260) * U * (G @ np.abs(wg) + V @ np.abs(wu))
    bg = edg.T @ np.abs(x) + (t + 8) * U * (G.T @ np.abs(x))
    bu = edu.T @ np.abs(x) + (t + 8) * U * (V.T @ np.abs(x))
    return [(w, b + H * (np.abs(w) + b)) for w, b in ((dx, bx), (dwg, bg), (dwu, bu))]


@pytest.mark.parametrize("fmt", [R.NV, R.MX])
@pytest.mark.parametrize("act", [0, 1])
@pytest.mark.parametrize("t,f,d", [(1, 1, 32), (9, 129, 96), (64, 128, 256), (130, 257, 416), (257, 300, 1056)])
def test_gated_backward(B, fmt, act, t, f, d):
    x, wg, wu = gated_operands(t, f, d, fmt)
    dh = bf16(np.random.default_rng(4).standard_normal((t, f)))
    ws = torch.empty(B.fp4_gated_ff_backward_workspace(t, f, d), dtype=torch.uint8, device=DEV)
    dx, c0 = guarded(t, d, torch.bfloat16)
    dg, c1 = guarded(f, d, torch.bfloat16)
    du, c2 = guarded(f, d, torch.bfloat16)
    h, c3 = guarded(t, f, torch.bfloat16)
    B.fp4_gated_ff_backward(fmt, act, x.op, wg.op, wu.op, dh.to(DEV), dx, dg, du, h, ws)
    bounds = grad_bounds(act, x.v, wg.v, wu.v, dh.double().numpy(), d)
    for got, (want, bound), what in zip((dx, dg, du), bounds, ("dx", "dgate", "dup")):
        near(got, want, bound, what)
    for c in (c0, c1, c2, c3):
        c()
    fwd = torch.empty_like(h)
    B.fp4_gated_ff(fmt, act, x.op, wg.op, wu.op, fwd)
    assert torch.equal(h, fwd)                                   # the forward call's result, bit for bit
    only = torch.empty_like(dx)
    B.fp4_gated_ff_backward(fmt, act, x.op, wg.op, wu.op, dh.to(DEV), only, None, None, None, ws)
    assert torch.equal(only, dx)
    g2, u2 = torch.empty_like(dg), torch.empty_like(du)
    wide = torch.zeros(t, f + 3, dtype=torch.bfloat16, device=DEV)
    wide[:, 1:1 + f] = dh.to(DEV)
    B.fp4_gated_ff_backward(fmt, act, x.op, wg.op, wu.op, wide[:, 1:1 + f], None, g2, u2, None, ws)
    assert torch.equal(g2, dg) and torch.equal(u2, du)


@pytest.mark.parametrize("act", [0, 1])
def test_gated_backward_against_differences(B, act):
    """Along random directions, central differences of sum(dh * h) in 64 bits (their own error, of
    order step^2, is below 1e-6 here) against the gradients' inner products with the direction; the
    bound is the gradients' own, entry by entry."""
    t, f, d = 24, 70, 128
    x, wg, wu = gated_operands(t, f, d, R.NV)
    dh = bf16(np.random.default_rng(4).standard_normal((t, f)))
    D = dh.double().numpy()
    ws = torch.empty(B.fp4_gated_ff_backward_workspace(t, f, d), dtype=torch.uint8, device=DEV)
    grads = [torch.empty(*s, dtype=torch.bfloat16, device=DEV) for s in ((t, d), (f, d), (f, d))]
    B.fp4_gated_ff_backward(R.NV, act, x.op, wg.op, wu.op, dh.to(DEV), *grads, None, ws)
    bounds = grad_bounds(act, x.v, wg.v, wu.v, D, d)
    g = np.random.default_rng(8)
    for i, grad in enumerate(grads):
        for _ in range(4):
            at = [x.v, wg.v, wu.v]
            v = g.standard_normal(at[i].shape)
            step = 1e-5

            def loss(s):
                p = list(at)
                p[i] = p[i] + s * v
                return (D * R.gated(act, *p)).sum()
            diff = (loss(step) - loss(-step)) / (2 * step)
            assert abs((host(grad) * v).sum() - diff) <= (bounds[i][1] * np.abs(v)).sum() + 1e-6 * abs(diff) + 1e-6


def test_matmul_backward_against_differences(B):
    m, n, k = 20, 45, 96
    a, b = Held(m, k, R.MX, 1), Held(n, k, R.MX, 2)
    dD = bf16(np.random.default_rng(4).standard_normal((m, n)))
    d = dD.double().numpy()
    ws = torch.empty(B.fp4_matmul_backward_workspace(m, n, k), dtype=torch.uint8, device=DEV)
    dA, dB = (torch.empty(r, k, dtype=torch.bfloat16, device=DEV) for r in (m, n))
    B.fp4_matmul_backward(R.MX, a.op, b.op, dD.to(DEV), dA, dB, ws)
    v = np.random.default_rng(5).standard_normal((m, k))
    w = np.random.default_rng(6).standard_normal((n, k))
    for grad, diff, u in ((dA, (d * ((a.v + v) @ b.v.T - (a.v - v) @ b.v.T)).sum() / 2, v),
                          (dB, (d * (a.v @ (b.v + w).T - a.v @ (b.v - w).T)).sum() / 2, w)):
        scale = np.abs(d) @ np.abs(b.v) if u is v else np.abs(d).T @ np.abs(a.v)
        bound = H * np.abs(host(grad)) * (1 + 2 * H) + (n + 4) * U * scale
        assert abs((host(grad) * u).sum() - diff) <= (bound * np.abs(u)).sum() + 1e-9 * abs(diff)


@pytest.mark.parametrize("power", [0, 60, 100])
def test_gated_backward_far_from_zero(B, power):
    """Gates of +-64 * 36 * 2^power, whose square overflows fp32 for the larger two: act' is 1 or 0 there.
    g is exact in fp32 and act adds nothing to it, so each gradient is the sum of exact terms after one
    rounding of dg or du to bf16 (u's own error is within the few U beside it)."""
    t, f, d = 5, 40, 64
    wu = Held(f, d, R.MX, 3, 0)
    wg = np.full((f, d // 2), 0x77, np.uint8)                    # 6 in every place
    wg[20:] = 0xFF                                               # -6
    sx, sg = np.full((t, d // 32), 127, np.uint8), np.full((f, d // 32), 127 + power, np.uint8)
    x, gate = ((torch.from_numpy(c).to(DEV), torch.from_numpy(R.swizzle(s)).to(DEV), None)
               for c, s in ((np.full((t, d // 2), 0x77, np.uint8), sx), (wg, sg)))
    vx, vg = np.full((t, d), 6.0), R.values(wg, sg, R.MX)
    g, u = vx @ vg.T, vx @ wu.v.T
    on = (g > 0).astype(np.float64)
    dh = bf16(np.random.default_rng(4).standard_normal((t, f)))
    D = dh.double().numpy()
    dg, du = D * u * on, D * g * on
    ws = torch.empty(B.fp4_gated_ff_backward_workspace(t, f, d), dtype=torch.uint8, device=DEV)
    for act in (0, 1):
        got = [torch.empty(r, d, dtype=torch.bfloat16, device=DEV) for r in (t, f, f)]
        B.fp4_gated_ff_backward(R.MX, act, x, gate, wu.op, dh.to(DEV), *got, None, ws)
        su = np.abs(vx) @ np.abs(wu.v).T                         # what u's rounding is relative to
        for out, want, s, n in zip(got, (dg @ vg + du @ wu.v, dg.T @ vx, du.T @ vx),
                                   ((np.abs(D) * su * on) @ np.abs(vg) + np.abs(du) @ np.abs(wu.v),
                                    (np.abs(D) * su * on).T @ vx, np.abs(du).T @ vx), (2 * f, t, t)):
            near(out, want, (1 + 2 * H) * (H + (n + d + 16) * U) * s + H * np.abs(want) + 1e-30)


@pytest.mark.parametrize("t", [3, 130])
def test_gated_with_a_zero_weight(B, t):
    """A gate of zeros, whose global scale is 0 as nvfp4_global_scale gives it: h and d_x are zero, and the
    gate's own gradient is not lost."""
    f, d = 160, 96
    x, wg, wu = gated_operands(t, f, d, R.NV)
    S = torch.zeros(1, device=DEV)
    zero = (torch.zeros_like(wg.op[0]), torch.zeros_like(wg.op[1]), S)
    h = torch.empty(t, f, dtype=torch.bfloat16, device=DEV)
    B.fp4_gated_ff(R.NV, 0, x.op, zero, wu.op, h)
    assert not bool(h.any())
    dh = bf16(np.random.default_rng(4).standard_normal((t, f)))
    ws = torch.empty(B.fp4_gated_ff_backward_workspace(t, f, d), dtype=torch.uint8, device=DEV)
    dx, dg, du = (torch.empty(r, d, dtype=torch.bfloat16, device=DEV) for r in (t, f, f))
    B.fp4_gated_ff_backward(R.NV, 0, x.op, zero, wu.op, dh.to(DEV), dx, dg, du, None, ws)
    for got, (want, bound) in zip((dx, dg, du), grad_bounds(0, x.v, 0 * wg.v, wu.v, dh.double().numpy(), d)):
        near(got, want, bound)
    assert bool(dg.any()) and not bool(dx.any()) and not bool(du.any())


@pytest.mark.parametrize("fmt", [R.NV, R.MX])
def test_gradients_over_nothing_are_zero(B, fmt):
    """No tokens: the weights' gradients are sums over no rows; no columns: the tokens' are.  No workspace, the
    tensors without elements null or None."""
    none = lambda cols: (torch.empty(0, cols // 2, dtype=torch.uint8, device=DEV), torch.empty(0, dtype=torch.uint8, device=DEV), None)
    empty = lambda *s: torch.empty(*s, dtype=torch.bfloat16, device=DEV)
    w, up = Held(45, 96, fmt, 1), Held(45, 96, fmt, 2)
    for rows, a, b, dA_first in ((45, none(96), w.op, False), (45, w.op, none(96), True)):
        got, check = guarded(rows, 96, torch.bfloat16, 101, 1)
        grads = (got, empty(0, 96)) if dA_first else (empty(0, 96), got)
        d = empty(rows, 0) if dA_first else empty(0, rows)
        for other in (grads, tuple(g if g is got else None for g in grads)):
            got.fill_(3.0)
            B.fp4_matmul_backward(fmt, a, b, d, *other)
            assert not bool(got.any())
            check()
    (dg, cg), (du, cu) = (guarded(45, 96, torch.bfloat16, 104) for _ in range(2))
    for dx in (empty(0, 96), None):
        dg.fill_(3.0), du.fill_(3.0)
        B.fp4_gated_ff_backward(fmt, 0, none(96), w.op, up.op, empty(0, 45), dx, dg, du)
        assert not bool(dg.any()) and not bool(du.any())
        cg(), cu()
    B.fp4_gated_ff_backward(fmt, 0, none(96), w.op, up.op, empty(0, 45), empty(0, 96))      # frozen weights: nothing to write
    dx, check = guarded(45, 96, torch.bfloat16, 97)
    B.fp4_gated_ff_backward(fmt, 1, w.op, none(96), none(96), empty(45, 0), dx, empty(0, 96), empty(0, 96))
    assert not bool(dx.any())
    check()


# ------------------------------------------------------------------ use
def test_results_do_not_change_from_run_to_run(B):
    """Split sums are added in a fixed order: the same bits every time."""
    a, b = Held(3, 4096, R.NV, 1), Held(512, 4096, R.NV, 2)
    first = torch.empty(3, 512, device=DEV)
    B.fp4_matmul(R.NV, a.op, b.op, first)
    for _ in range(20):
        D = torch.empty_like(first)
        B.fp4_matmul(R.NV, a.op, b.op, D)
        assert torch.equal(D, first)


def test_on_another_stream_and_in_a_graph(B):
    t, f, d = 40, 256, 512
    x, wg, wu = gated_operands(t, f, d, R.MX)
    down = Held(96, f, R.MX, 9, 1)
    xin = torch.randn(t, d, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).to(DEV)
    codes = torch.empty(t, d // 2, dtype=torch.uint8, device=DEV)
    sf = torch.empty(B.mx_swizzled_bytes(t, d), dtype=torch.uint8, device=DEV)
    hc = torch.empty(t, f // 2, dtype=torch.uint8, device=DEV)
    hs = torch.empty(B.mx_swizzled_bytes(t, f), dtype=torch.uint8, device=DEV)
    y = torch.empty(t, 96, device=DEV)

    def step(stream=None):
        B.mxfp4_quantize(xin, codes, None, sf, stream=stream)
        B.fp4_gated_ff(R.MX, 0, (codes, sf, None), wg.op, wu.op, None, hc, hs, stream=stream)
        B.fp4_matmul(R.MX, (hc, hs, None), down.op, y, stream=stream)
    step()
    torch.cuda.synchronize()
    want = y.clone()
    s = torch.cuda.Stream()
    y.zero_()
    torch.cuda.synchronize()
    step(s)
    s.synchronize()
    assert torch.equal(y, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    y.zero_()
    xin.mul_(2.0)                                                # powers of two pass through every scale but the gate's
    graph.replay()
    torch.cuda.synchronize()
    got = y.clone()
    step()
    torch.cuda.synchronize()
    assert torch.equal(got, y) and not torch.equal(got, want)


def test_many_calls_back_to_back(B):
    """Calls of different sizes without a wait between them, each into its own output."""
    ops = [(Held(m, 512, R.NV, m), Held(n, 512, R.NV, n)) for m, n in ((1, 300), (70, 64), (260, 520), (16, 128))]
    outs = []
    for _ in range(10):
        for a, b in ops:
            D = torch.empty(a.v.shape[0], b.v.shape[0], device=DEV)
            B.fp4_matmul(R.NV, a.op, b.op, D)
            outs.append((a, b, D))
    torch.cuda.synchronize()
    for a, b, D in outs:
        near(D, a.v @ b.v.T, sum_bound(a.v, b.v, 512))


# ------------------------------------------------------------------ long contractions, split over pairs of CTAs
@pytest.mark.parametrize("fmt", [R.NV, R.MX])
@pytest.mark.parametrize("m,n,k", [(65, 129, 8224), (300, 1000, 8192), (257, 4100, 8960), (512, 4864, 8192)])
def test_matmul_long_contraction(B, fmt, m, n, k):
    a, b = Held(m, k, fmt, 5), Held(n, k, fmt, 6)
    for out in (torch.float32, torch.bfloat16):
        D, check = guarded(m, n, out)
        B.fp4_matmul(fmt, a.op, b.op, D)
        want = a.v @ b.v.T
        near(D, want, sum_bound(a.v, b.v, k) + (H * np.abs(want) if out == torch.bfloat16 else 0))
        check()


@pytest.mark.parametrize("fmt", [R.NV, R.MX])
@pytest.mark.parametrize("t,f,d", [(70, 192, 8224), (300, 416, 8192), (260, 2080, 8192)])
def test_gated_long_contraction(B, fmt, t, f, d):
    x, wg, wu = gated_operands(t, f, d, fmt)
    h, check = guarded(t, f, torch.bfloat16)
    codes = torch.full((t, f // 2), 0xAA, dtype=torch.uint8, device=DEV)
    sf = torch.full((B.mx_swizzled_bytes(t, f),), 0xAA, dtype=torch.uint8, device=DEV)
    B.fp4_gated_ff(fmt, 0, x.op, wg.op, wu.op, h, codes, sf)
    want, bound, *_ = gated_bounds(0, x.v, wg.v, wu.v, d)
    near(h, want, bound + H * (np.abs(want) + bound) + 2.0 ** -133)
    check()
    qc, _, qs, _ = quantised(B, h)
    assert torch.equal(codes, qc) and torch.equal(sf, qs)


@pytest.mark.parametrize("t,f,d", [(40, 1100, 8224), (2100, 72, 96)])
def test_gated_backward_long_sums(B, t, f, d):
    """Recomputed sums over d, sums over 2 f for d_x and over t for the weights, each past 32 stages of K."""
    x, wg, wu = gated_operands(t, f, d, R.NV)
    dh = bf16(np.random.default_rng(4).standard_normal((t, f)))
    ws = torch.empty(B.fp4_gated_ff_backward_workspace(t, f, d), dtype=torch.uint8, device=DEV)
    out = [guarded(r, d, torch.bfloat16) for r in (t, f, f)]
    B.fp4_gated_ff_backward(R.NV, 0, x.op, wg.op, wu.op, dh.to(DEV), *(o[0] for o in out), None, ws)
    for (got, check), (want, bound) in zip(out, grad_bounds(0, x.v, wg.v, wu.v, dh.double().numpy(), d)):
        near(got, want, bound)
        check()


# ------------------------------------------------------------------ offsets past 32 bits
def test_offsets_past_32_bits_in_the_result(B):
    m = n = 66000                                                # 4.4e9 elements
    a, b = Held(m, 32, R.MX, 1), Held(n, 32, R.MX, 2)
    D = torch.empty(m, n, dtype=torch.bfloat16, device=DEV)
    B.fp4_matmul(R.MX, a.op, b.op, D)
    for r in (0, 1, 33000, 65279, 65280, m - 1):
        want = a.v[r:r + 1] @ b.v.T
        near(D[r:r + 1], want, 36 * U * (np.abs(a.v[r:r + 1]) @ np.abs(b.v).T) + H * np.abs(want))


def test_offsets_past_32_bits_in_a_weight(B):
    n, k = 4300000, 2048                                         # 4.4e9 bytes of codes
    g = torch.Generator(device=DEV).manual_seed(1)
    codes = torch.randint(0, 256, (n, k // 2), dtype=torch.uint8, device=DEV, generator=g)
    sf = torch.randint(124, 131, (B.mx_swizzled_bytes(n, k),), dtype=torch.uint8, device=DEV, generator=g)
    for m in (1, 130):
        a = Held(m, k, R.MX, 3)
        D = torch.empty(m, n, device=DEV)
        B.fp4_matmul(R.MX, a.op, (codes, sf, None), D)
        for r0 in (0, n // 2 // 128 * 128, (n - 1) // 128 * 128):
            rows = min(128, n - r0)
            kb = k // 32
            r, c = np.meshgrid(np.arange(rows), np.arange(kb), indexing="ij")
            at = (r0 // 128 * (kb // 4) + c // 4) * 512 + (r % 32) * 16 + r // 32 * 4 + c % 4
            v = R.values(codes[r0:r0 + rows].cpu().numpy(), sf[torch.from_numpy(at).to(DEV)].cpu().numpy(), R.MX)
            near(D[:, r0:r0 + rows], a.v @ v.T, sum_bound(a.v, v, k))


def test_offsets_past_32_bits_in_quantisation(B):
    rows, cols = 270000, 65536                                   # 1.8e10 elements: past a launch's 2^30 segments
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device=DEV)
    at = [0, 1, 65535, 131071, 262143, 262144, 262145, rows - 1]
    x[at] = torch.randn(len(at), cols, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).to(DEV)
    codes = torch.full((rows, cols // 2), 0xAA, dtype=torch.uint8, device=DEV)
    sf = torch.full((rows, cols // 32), 0xAA, dtype=torch.uint8, device=DEV)
    B.mxfp4_quantize(x, codes, sf)
    wc, ws = R.mxfp4(host(x[at]))
    assert np.array_equal(codes[at].cpu().numpy(), wc) and np.array_equal(sf[at].cpu().numpy(), ws)
    others = [2, 100000, 262143 - 7, 262150]
    assert not bool(codes[others].any()) and not bool(sf[others].any())
    del x
    out = torch.empty(rows, cols, dtype=torch.bfloat16, device=DEV)
    B.mxfp4_dequantize(codes, sf, B.NVFP4_SF_LINEAR, rows, cols, out)
    assert np.array_equal(host(out[at]), R.values(wc, ws, R.MX)) and not bool(out[others].any())


# one CTA to a tile, a cluster of them, pairs over several tiles, pairs that split K
@pytest.mark.parametrize("m,n,k", [(3, 10000, 512), (3, 256, 4096), (300, 600, 512), (200, 256, 8192)])
def test_waits_that_run_out_are_reported(B, m, n, k):
    """The status word says so, the output is untouched and the next call is right."""
    a, b = Held(m, k, R.NV, 1), Held(n, k, R.NV, 2)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    D = torch.full((m, n), 7.0, device=DEV)
    B.fp4_selftest_wait_timeout(R.NV, a.op, b.op, D, st)
    torch.cuda.synchronize()
    assert st.item() == 16 and bool((D == 7.0).all())
    st.zero_()
    B.fp4_matmul(R.NV, a.op, b.op, D, st)
    near(D, a.v @ b.v.T, sum_bound(a.v, b.v, k))
    assert st.item() == 0
