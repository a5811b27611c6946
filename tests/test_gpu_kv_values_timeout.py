"""Attention's bounded waits: where the values of the last keys do not come, no row is written without them."""
import time

import pytest
import torch

import kv_plans as P
import kv_reference as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2606_07618_gb300 import binding
    binding.lib()
    return binding


# sequences of one tile of keys, whose scores are all there when the wait runs out, and longer ones
@pytest.mark.parametrize("shape,path", [(([40, 90], [30, 20], 38, 3, 64, 16), 256), (([40, 90, 128], [30, 20, 128], 76, 2, 128, 16), 256),
                                        (([300, 1000], [90, 100], 38, 3, 64, 16), 256), (([120, 2100], [165, 170], 39, 3, 128, 32), 512)])
def test_values_that_do_not_come(B, shape, path):
    s = R.Setting(*shape, seed=11)
    assert P.path_of(s) == (path, "alone", 0)
    n, b = max(s.queries), len(s.lens)
    dev = [t.cuda() for t in s.cache]
    q, out = s.q.cuda(), torch.full_like(s.q, 7.0, device="cuda")
    table, lens, offsets = s.table.cuda(), torch.tensor(s.lens, dtype=torch.int32, device="cuda"), s.offsets.cuda()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    assert B.nvfp4_kv_attention_workspace(dev, q, b, table.shape[1], n) == 0
    torch.cuda.synchronize()
    t0 = time.time()
    B.nvfp4_kv_selftest_wait_timeout(q, dev, table, lens, offsets, n, s.scale, out, status, values=True)
    torch.cuda.synchronize()
    assert 0.5 < time.time() - t0 < 60
    assert status.item() == 16 and (out == 7.0).all()
    out, lse = s.run(B)
    R.check(out, s.want(), lse)
