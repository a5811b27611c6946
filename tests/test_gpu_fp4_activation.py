"""The gated feed-forward where the activation is next to nothing: act(g) keeps its relative accuracy down to fp32's
smallest numbers, which a large u or dh brings back into range.

Gates and u are exact in fp32.  The activation is g p with p = e / (1 + e), e = exp(z): CUDA documents 2 + |1.173 z|
units of 2^-23 for the fast exponential, less than 2^-16 for |z| < 104, and z itself (GELU's) is off by at most five
roundings of 2^-24 of 104, 2^-15; the quotient and products are a few units more: 2^-14 in all.  Below 2^-126
e and p are multiples of 2^-149.  One H = 2^-8 for each rounding to bf16."""
import numpy as np
import pytest
import torch

import fp4_reference as R

pytestmark = pytest.mark.gpu
DEV = "cuda"
U, H, A = 2.0 ** -23, 2.0 ** -8, 2.0 ** -14


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2606_07618_gb300 import binding
    binding.lib()
    return binding


def held(codes, sf):
    return torch.from_numpy(codes).to(DEV), torch.from_numpy(R.swizzle(sf)).to(DEV), None


def rows_of_sum(sums, step):
    """[len(sums), 32] E2M1 codes whose values times 2 step add up to each sum, a multiple of step."""
    out = np.zeros((len(sums), 32), np.uint8)
    for r, s in enumerate(sums):
        left = abs(s) / (2 * step)
        for k in range(32):
            c = int(np.searchsorted(R.GRID, left, side="right")) - 1
            out[r, k] = c | (8 if s < 0 else 0)
            left -= R.GRID[c]
        assert left == 0
    return out[:, 0::2] | (out[:, 1::2] << 4)


def case(act):
    """Gates from where exp(z) is 2^-80 to where it is 2^-149, and the activation and its derivative there."""
    step = 0.5 if act == 0 else 2.0 ** -5
    g = -np.arange(56, 103, step) if act == 0 else -np.arange(8.5, 10.65, step)
    z, dz = (g, 1.0) if act == 0 else (2 * np.sqrt(2 / np.pi) * (g + 0.044715 * g ** 3),
                                       2 * np.sqrt(2 / np.pi) * (1 + 3 * 0.044715 * g * g))
    p = np.exp(z) / (1 + np.exp(z))
    assert z.min() < -100 and np.abs(z).max() < 104
    return g, step, p, g * p, p + g * p * (1 - p) * dz, dz


@pytest.mark.parametrize("act", [0, 1])
@pytest.mark.parametrize("t", [3, 40, 300])
def test_small_activations(B, act, t):
    g, step, p, a, da, dz = case(act)
    f, d = len(g), 32
    x = held(np.full((t, 16), 0x22, np.uint8), np.full((t, 1), 127, np.uint8))               # ones
    gate = held(rows_of_sum(g, step), np.full((f, 1), 127 + int(np.log2(2 * step)), np.uint8))
    cu = np.zeros((f, 16), np.uint8)
    cu[:, 0] = 0x02
    up = held(cu, np.full((f, 1), 127 + 60, np.uint8))                                       # u = 2^60
    h = torch.empty(t, f, dtype=torch.bfloat16, device=DEV)
    B.fp4_gated_ff(R.MX, act, x, gate, up, h)
    tiny = 2.0 ** -148 * np.abs(g)                               # e and p: half a unit each, and what follows from them
    want, bound = a * 2.0 ** 60, (A + H) * np.abs(a) * 2.0 ** 60 + tiny * 2.0 ** 60
    got = h.double().cpu().numpy()
    assert (np.abs(got - want) <= bound).all(), np.flatnonzero((np.abs(got - want) > bound).any(0))
    dh = torch.full((t, f), 2.0 ** 30, dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(B.fp4_gated_ff_backward_workspace(t, f, d), dtype=torch.uint8, device=DEV)
    dg, du = (torch.empty(f, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    B.fp4_gated_ff_backward(R.MX, act, x, gate, up, dh, None, dg, du, h, ws)
    got = h.double().cpu().numpy()
    assert (np.abs(got - want) <= bound).all()
    # t equal rows: sums of t equal terms; act' is p + a (1 - p) z', two terms of which the larger bounds the error
    r = A + 2 * H + (t + 8) * U
    for out, want, err in ((du, a * t * 2.0 ** 30, r * np.abs(a) + tiny),
                           (dg, da * t * 2.0 ** 90, r * (p + np.abs(a) * dz) + tiny * (1 + dz))):
        scale = np.abs(want / np.where(out is du, a, da))
        got = out.double().cpu().numpy()
        assert (np.abs(got - want[:, None]) <= (err * scale)[:, None]).all()
