"""The feed-forward block of feed_forward.py end to end: each stage against 64 bits on the operands it
was given, in either format, and the refusals."""
import numpy as np
import pytest
import torch

import fp4_reference as R

pytestmark = pytest.mark.gpu
DEV = "cuda"
U, H = 2.0 ** -23, 2.0 ** -8


@pytest.fixture(scope="module")
def F():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2606_07618_gb300 import feed_forward
    return feed_forward


def value(op, fmt):
    """The values of an operand, its scales read from the 128x4-atom layout."""
    codes, sf = op[0].cpu().numpy(), op[1].cpu().numpy()
    rows, kb = codes.shape[0], 2 * codes.shape[1] // R.block_of(fmt)
    r, k = np.meshgrid(np.arange(rows), np.arange(kb), indexing="ij")
    at = ((r // 128) * -(-kb // 4) + k // 4) * 512 + (r % 32) * 16 + (r // 32) % 4 * 4 + k % 4
    return R.values(codes, sf[at], fmt, 1.0 if op[2] is None else op[2].item())


def block(F, fmt, f, d, seed=1, act=0):
    g = torch.Generator().manual_seed(seed)
    w = [(s[1] ** -0.5 * torch.randn(*s, generator=g)).to(torch.bfloat16).to(DEV) for s in ((f, d), (f, d), (d, f))]
    return F.GatedFeedForward(*w, fmt=fmt, act=act), w


@pytest.mark.parametrize("fmt", [R.NV, R.MX])
@pytest.mark.parametrize("act", [0, 1])
@pytest.mark.parametrize("t,f,d", [(1, 96, 64), (33, 160, 128), (200, 416, 256)])
def test_block(F, fmt, act, t, f, d):
    ff, w = block(F, fmt, f, d, act=act)
    x = torch.randn(t, d, generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).to(DEV)
    y = ff(x)
    dy = torch.randn(t, d, generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).to(DEV)
    g = ff.backward(dy)
    torch.cuda.synchronize()
    assert ff.status.item() == 0
    vx, vg, vu, vd, vh = (value(o, fmt) for o in (ff._x, ff.gate, ff.up, ff.down, ff._h))
    # quantised values are within half of the widest step of their grid: 1/6 of a block's maximum (a scale
    # may round down by 1/16 more in NVFP4, or by a factor of two in MXFP4, where 6 to 8 go to 6)
    for v, of in ((vx, x), (vg, w[0]), (vu, w[1]), (vd, w[2])):
        o = of.double().cpu().numpy()
        top = np.abs(o.reshape(o.shape[0], -1, R.block_of(fmt))).max(-1).repeat(R.block_of(fmt), 1)
        assert (np.abs(v - o) <= 0.26 * top + 1e-12).all()
    want = vh @ vd.T
    y = y.double().cpu().numpy()
    assert (np.abs(y - want) <= (f + 4) * U * (np.abs(vh) @ np.abs(vd).T) + H * np.abs(want)).all()
    dyn = dy.double().cpu().numpy()
    dd = dyn.T @ vh
    assert (np.abs(g["down"].double().cpu().numpy() - dd) <= (t + 4) * U * (np.abs(dyn).T @ np.abs(vh)) + H * np.abs(dd)).all()
    # dh is rounded to bf16 before the gated part takes it, then dg and du: four roundings in a row at most
    dh = dyn @ vd
    a, da = R.act(act, vx @ vg.T)
    u = vx @ vu.T
    sx = np.abs(dh * u * da) @ np.abs(vg) + np.abs(dh * a) @ np.abs(vu)
    sg, su = np.abs(dh * u * da).T @ np.abs(vx), np.abs(dh * a).T @ np.abs(vx)
    for got, ref, s in zip((g["x"], g["gate"], g["up"]), R.gated_grad(act, vx, vg, vu, dh), (sx, sg, su)):
        # 2^-14 |dh| covers what rounding g and u to fp32 sums makes of the factors (|g|, |u| of a few units)
        assert (np.abs(got.double().cpu().numpy() - ref) <= 4 * H * s + H * np.abs(ref) + 2.0 ** -14 * np.abs(dh).max() * np.abs(s).max()).all()
    only = ff.backward(dy, weights=False)
    assert list(only) == ["x"] and torch.equal(only["x"], g["x"])


@pytest.mark.parametrize("fmt", [R.NV, R.MX])
def test_no_tokens(F, fmt):
    """An empty batch: an empty result, and gradients of zeros for the weights."""
    ff, _ = block(F, fmt, 96, 64)
    none = torch.empty(0, 64, dtype=torch.bfloat16, device=DEV)
    assert ff(none).shape == (0, 64)
    g = ff.backward(none)
    assert g["x"].shape == (0, 64) and all(not bool(g[n].any()) for n in ("gate", "up", "down"))
    assert list(ff.backward(none, weights=False)) == ["x"] and int(ff.status) == 0


def test_nvfp4_weights_are_scalesweeps(F):
    """The block's NVFP4 weights are the grouped ScaleSweep's, bit for bit."""
    from paper_2606_07618_gb300 import binding as B
    from paper_2606_07618_gb300.step import QuantizeStep
    ff, w = block(F, R.NV, 128, 64)
    q = QuantizeStep(w)
    q()
    for o, op in zip(q.outs, (ff.gate, ff.up, ff.down)):
        assert torch.equal(o["codes"], op[0]) and torch.equal(o["sf_swizzled"], op[1])
    imp = [torch.rand(n, device=DEV) + 0.1 for n in (64, 64, 128)]
    weighted = F.GatedFeedForward(*w, fmt=B.FP4_FMT_NVFP4, importance=imp)
    assert not torch.equal(weighted.gate[0], ff.gate[0])


def test_refusals(F):
    _, w = block(F, R.MX, 64, 32)
    with pytest.raises(ValueError):
        F.GatedFeedForward(w[0], w[1], w[0])
    with pytest.raises(ValueError):
        F.GatedFeedForward(*w, fmt=5)
    with pytest.raises(ValueError):
        F.GatedFeedForward(*w, fmt=R.MX, importance=[None] * 3)
    with pytest.raises(ValueError):
        F.GatedFeedForward(w[0][:50], w[1][:50], w[2][:, :50])
    ff, _ = block(F, R.MX, 64, 32)
    with pytest.raises(RuntimeError):
        ff.backward(torch.zeros(1, 32, dtype=torch.bfloat16, device=DEV))
    with pytest.raises(ValueError):
        ff(torch.zeros(4, 64, dtype=torch.bfloat16, device=DEV))
    ff(torch.zeros(4, 32, dtype=torch.bfloat16, device=DEV))
    with pytest.raises(ValueError):
        ff.backward(torch.zeros(5, 32, dtype=torch.bfloat16, device=DEV))
