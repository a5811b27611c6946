"""Dense tensors of the 4-bit calls that are columns of one buffer: accepted where their columns lie beside each other,
with the results of tensors of their own, and refused where they share some."""
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


def held(rows, cols, seed, spread=1):
    codes, sf, S = R.random_matrix(rows, cols, R.NV, seed, spread)
    return torch.from_numpy(codes).to(DEV), torch.from_numpy(R.swizzle(sf)).to(DEV), torch.tensor([S], device=DEV)


def bf16(rows, cols, seed):
    return torch.from_numpy(np.random.default_rng(seed).standard_normal((rows, cols)).astype(np.float32)).to(torch.bfloat16).to(DEV)


def empty(*s):
    return torch.empty(*s, dtype=torch.bfloat16, device=DEV)


@pytest.mark.parametrize("d", [64, 160])
def test_both_weight_gradients_in_one_buffer(B, d):
    t, f = 70, 200
    ops = held(t, d, 1), held(f, d, 2), held(f, d, 3)
    dh, ws = bf16(t, f, 4), torch.empty(B.fp4_gated_ff_backward_workspace(t, f, d), dtype=torch.uint8, device=DEV)
    want = empty(t, d), empty(f, d), empty(f, d)
    B.fp4_gated_ff_backward(0, 0, *ops, dh, *want, None, ws)
    whole, dx = torch.full((f + 1, 2 * d + 8), 7.0, dtype=torch.bfloat16, device=DEV), empty(t, d)
    both = whole[:f]
    B.fp4_gated_ff_backward(0, 0, *ops, dh, dx, both[:, :d], both[:, d:2 * d], None, ws)
    assert torch.equal(dx, want[0]) and torch.equal(both[:, :d], want[1]) and torch.equal(both[:, d:2 * d], want[2])
    assert bool((both[:, 2 * d:] == 7.0).all()) and bool((whole[f] == 7.0).all())
    for a, b in ((both[:, :d], both[:, d - 1:2 * d - 1]), (both[:, 8:d + 8], both[:, :d]), (both[:, :d], both[:, :d])):
        with pytest.raises(B.Nvfp4Error):
            B.fp4_gated_ff_backward(0, 0, *ops, dh, dx, a, b, None, ws)
    wraps = whole.view(-1)[d + 9:d + 9 + f * (2 * d + 8)].view(f, -1)[:, :d]     # a row's last column is in the next row
    with pytest.raises(B.Nvfp4Error):
        B.fp4_gated_ff_backward(0, 0, *ops, dh, dx, both[:, :d], wraps, None, ws)


def test_a_result_beside_the_gradient_it_is_formed_from(B):
    """d_out and the two gradients in columns of buffers they share, h beside dh, a status word in a gap."""
    m, n, k = 40, 72, 96
    a, b = held(m, k, 1), held(n, k, 2)
    ws = torch.empty(B.fp4_matmul_backward_workspace(m, n, k), dtype=torch.uint8, device=DEV)
    buf = torch.zeros(m, 192, dtype=torch.bfloat16, device=DEV)
    buf[:, 8:80] = bf16(m, n, 3)
    dA, dB = empty(m, k), empty(n, k)
    B.fp4_matmul_backward(0, a, b, buf[:, 8:80].contiguous(), dA, dB, ws)
    other = empty(n, k)
    B.fp4_matmul_backward(0, a, b, buf[:, 8:80], buf[:, 96:192], other, ws)
    assert torch.equal(buf[:, 96:192], dA) and torch.equal(other, dB)
    with pytest.raises(B.Nvfp4Error):
        B.fp4_matmul_backward(0, a, b, buf[:, 8:80], buf[:, 79:175], other, ws)
    wide = torch.full((m, 128), 7.0, dtype=torch.float32, device=DEV)
    wide[5, 100] = 0
    status = wide.view(torch.int32)[5, 100:101]
    B.fp4_matmul(0, a, b, wide[:, :n], status)
    want = torch.empty(m, n, device=DEV)
    B.fp4_matmul(0, a, b, want)
    assert torch.equal(wide[:, :n], want) and status.item() == 0
    with pytest.raises(B.Nvfp4Error):
        B.fp4_matmul(0, a, b, wide[:, :n], wide.view(torch.int32)[5, n - 1:n])
