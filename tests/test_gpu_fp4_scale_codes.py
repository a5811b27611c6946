"""Every E8M0 scale code, from 2^-127 to 2^127 and NaN, through dequantisation, products and gradients.  Each sum is of
equal powers of two or of few of them, so results are exact."""
import numpy as np
import pytest
import torch

import fp4_reference as R

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2606_07618_gb300 import binding
    binding.lib()
    return binding


def held(codes, sf):
    return torch.from_numpy(codes).to(DEV), torch.from_numpy(R.swizzle(sf)).to(DEV), None


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_dequantise(B, dtype):
    codes = np.tile(np.arange(16, dtype=np.uint8) * 0x11, (256, 2))[:, :16]
    sf = np.arange(256, dtype=np.uint8)[:, None]
    with np.errstate(all="ignore"):
        want = torch.from_numpy(R.values(codes, sf, R.MX)).to(torch.float32).to(dtype)
    for layout, s in ((B.NVFP4_SF_LINEAR, sf), (B.NVFP4_SF_SWIZZLED, R.swizzle(sf))):
        out = torch.empty(256, 32, dtype=dtype, device=DEV)
        B.mxfp4_dequantize(torch.from_numpy(codes).to(DEV), torch.from_numpy(s.copy()).to(DEV), layout, 256, 32, out)
        assert torch.equal(torch.nan_to_num(out.cpu(), nan=-3.0, posinf=-5.0, neginf=-7.0),
                           torch.nan_to_num(want, nan=-3.0, posinf=-5.0, neginf=-7.0))


@pytest.mark.parametrize("rows", [np.array([0, 1, 2, 30, 100, 126, 127, 128, 150, 200, 252, 253, 254]), np.arange(255)])
def test_products(B, rows):
    """Ones with scales 2^(i - 127) and 2^(j - 127): 32 2^(i + j - 254) wherever fp32 has it as a normal number."""
    ones = lambda n: np.full((n, 16), 0x22, np.uint8)  # noqa: E731
    i, j = rows[:, None], np.arange(255)[None, :]
    D = torch.empty(len(rows), 255, device=DEV)
    B.fp4_matmul(R.MX, held(ones(len(rows)), rows.astype(np.uint8)[:, None]), held(ones(255), np.arange(255, dtype=np.uint8)[:, None]), D)
    e = i + j - 254 + 5
    want, there = np.ldexp(1.0, np.clip(e, -126, 127)), (e >= -126) & (e <= 127)
    got = D.double().cpu().numpy()
    assert there.any(0).all() and (got == want)[there].all(), np.argwhere((got != want) & there)[:8]
    nan = torch.empty(len(rows), 3, device=DEV)
    B.fp4_matmul(R.MX, held(ones(len(rows)), rows.astype(np.uint8)[:, None]), held(ones(3), np.array([[127], [255], [127]], np.uint8)), nan)
    assert bool(nan[:, 1].isnan().all()) and not bool(nan[:, ::2].isnan().any())


@pytest.mark.parametrize("q", [1, 2, 3, 4, 5, 6, 7])
def test_gradients(B, q):
    """dA[i] = sum_n dD[i, n] B[n], one n at a time: the value q 2^(n - 127) of row n, brought to a normal number by
    a dD of 2^(100, 0 or -100).  All values that fp32 has, which are those that mxfp4_quantize gives and more."""
    n = 255
    b = held(np.full((n, 16), q * 0x11, np.uint8), np.arange(n, dtype=np.uint8)[:, None])
    value = R.GRID[q] * np.ldexp(1.0, np.arange(n) - 127)
    power = np.where(np.arange(n) < 60, 100, np.where(np.arange(n) < 200, 0, -100))
    a = held(np.full((n, 16), 0x22, np.uint8), np.full((n, 1), 127, np.uint8))
    dD = torch.from_numpy(np.diag(np.ldexp(1.0, power)).astype(np.float32)).to(torch.bfloat16).to(DEV)
    ws = torch.empty(B.fp4_matmul_backward_workspace(n, n, 32), dtype=torch.uint8, device=DEV)
    dA, dB = (torch.empty(n, 32, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    finite = value < 2.0 ** 128                                  # 0 times an infinite one is NaN in every row of dA
    last = int(finite.sum())
    rows = held(np.full((last, 16), q * 0x11, np.uint8), np.arange(last, dtype=np.uint8)[:, None])
    B.fp4_matmul_backward(R.MX, a, rows, dD[:, :last].contiguous(), dA, None, ws)
    want = value * np.ldexp(1.0, power)
    assert last >= 253 and (dA[:last].double().cpu().numpy() == want[:last, None]).all()
    # and as the operand whose own gradient is the other's: dB[j] = sum_m dD[m, j] A[m]
    B.fp4_matmul_backward(R.MX, rows, a, dD[:last].contiguous(), None, dB, ws)
    assert (dB[:last].double().cpu().numpy() == want[:last, None]).all()
