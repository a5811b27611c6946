"""Tokens written into the NVFP4 cache and read back: the same codes as the library's quantisers give, in the right places."""
import pytest
import torch

import kv_reference as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2606_07618_gb300 import binding
    binding.lib()
    return binding


def empty_cache(pages, heads, page, dim, S=(0.013, 0.021), fill=0x55):
    return (torch.full((pages, heads, 2, page, dim // 2), fill, dtype=torch.uint8, device="cuda"),
            torch.full((pages, heads, 2, dim // 16, page), fill, dtype=torch.uint8, device="cuda"),
            torch.tensor([S[0]], device="cuda"), torch.tensor([S[1]], device="cuda"))


def tensors(tokens, heads, dim, dt, seed=1):
    g = torch.Generator().manual_seed(seed)
    return [(torch.randn(tokens, heads, dim, generator=g) * torch.exp(torch.randn(tokens, heads, 1, generator=g))).to(dt).cuda()
            for _ in range(2)]


def quantised(B, x, S, sweep):
    """Codes [tokens, heads, dim/2] and scale codes [tokens, heads, dim/16] of the library's own quantisers."""
    t, h, d = x.shape
    out = B.empty_outputs(t * h, d, 16)
    x = x.reshape(t * h, d).contiguous()
    if sweep:
        B.scalesweep_quantize(x, 16, S, B.NVFP4_OBJ_MSE, None, 0, B.NVFP4_WINDOW_DEFAULT, B.NVFP4_WINDOW_DEFAULT, out["codes"],
                              out["sf_linear"])
    else:
        B.absmax_quantize(x, 16, S, out["codes"], out["sf_linear"])
    return out["codes"].view(t, h, d // 2), out["sf_linear"].view(t, h, d // 16)


@pytest.mark.parametrize("sweep", [True, False])
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("tokens,heads,dim,page", [(1, 1, 64, 16), (9, 3, 128, 16), (130, 2, 64, 32), (77, 8, 128, 1024)])
def test_write_gives_the_quantisers_codes(B, sweep, dt, tokens, heads, dim, page):
    pages = -(-tokens // page) + 3
    cache = empty_cache(pages, heads, page, dim)
    before = [c.clone() for c in cache[:2]]
    k, v = tensors(tokens, heads, dim, dt)
    slots = torch.randperm(pages * page, generator=torch.Generator().manual_seed(2))[:tokens].cuda()
    if tokens > 4:
        slots[3] = -1                                            # padding
    B.nvfp4_kv_write(cache, k, v, slots, B.NVFP4_KV_SWEEP if sweep else B.NVFP4_KV_ABSMAX)
    for part, x in enumerate((k, v)):
        codes, sf = quantised(B, x, cache[2 + part], sweep)
        keep = slots >= 0
        at, off = slots[keep] // page, slots[keep] % page
        before[0][at, :, part, off] = codes[keep]
        before[1][at, :, part, :, off] = sf[keep]
    assert torch.equal(cache[0], before[0]) and torch.equal(cache[1], before[1])


@pytest.mark.parametrize("which", [0, 1])
def test_one_of_keys_and_values(B, which):
    cache = empty_cache(2, 2, 16, 64)
    both = empty_cache(2, 2, 16, 64)
    kv = tensors(20, 2, 64, torch.bfloat16)
    slots = torch.arange(20, device="cuda") + 5
    B.nvfp4_kv_write(both, *kv, slots)
    B.nvfp4_kv_write(cache, *(x if i == which else None for i, x in enumerate(kv)), slots)
    for c, b in zip(cache[:2], both[:2]):
        assert torch.equal(c[:, :, which], b[:, :, which]) and (c[:, :, 1 - which] == 0x55).all()
    table, offsets = torch.tensor([[0, 1]], dtype=torch.int32, device="cuda"), torch.tensor([0, 20], dtype=torch.int32, device="cuda")
    starts = torch.tensor([5], dtype=torch.int32, device="cuda")
    full, one = [torch.empty(20, 2, 64, device="cuda") for _ in range(2)], torch.empty(20, 2, 64, device="cuda")
    B.nvfp4_kv_read(both, table, starts, offsets, *full)
    B.nvfp4_kv_read(cache, table, starts, offsets, **{"kv"[which]: one})
    assert torch.equal(one, full[which])


def test_strides_of_a_projection(B):
    """Keys and values as columns of one buffer, an odd row stride and a base that is not 16-byte aligned among them."""
    heads, dim, tokens = 2, 64, 21
    for pad, first in ((0, 0), (8, 0), (1, 0), (0, 1)):
        g = torch.Generator().manual_seed(3)
        buf = torch.randn(tokens, 6 * heads * dim + pad + first, generator=g).to(torch.bfloat16).cuda()
        k, v = (buf[:, first + i * heads * dim:first + (i + 1) * heads * dim].unflatten(1, (heads, dim)) for i in (4, 5))
        a, b = empty_cache(2, heads, 16, dim), empty_cache(2, heads, 16, dim)
        slots = torch.arange(tokens, device="cuda")
        B.nvfp4_kv_write(a, k, v, slots)
        B.nvfp4_kv_write(b, k.contiguous(), v.contiguous(), slots)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
        table, offsets = torch.tensor([[0, 1]], dtype=torch.int32, device="cuda"), torch.tensor([0, tokens], dtype=torch.int32, device="cuda")
        want = [torch.empty(tokens, heads, dim, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        B.nvfp4_kv_read(a, table, None, offsets, *want)
        rest = buf[:, :first + 4 * heads * dim].clone()
        B.nvfp4_kv_read(a, table, None, offsets, k, v)           # into the projection's columns
        assert torch.equal(k, want[0]) and torch.equal(v, want[1]) and torch.equal(buf[:, :first + 4 * heads * dim], rest)
        # heads first
        kt = k.transpose(0, 1).contiguous().transpose(0, 1)
        c = empty_cache(2, heads, 16, dim)
        B.nvfp4_kv_write(c, kt, None, slots, B.NVFP4_KV_ABSMAX)
        B.nvfp4_kv_write(b, k.contiguous(), None, slots, B.NVFP4_KV_ABSMAX)
        assert torch.equal(c[0][:, :, 0], b[0][:, :, 0])


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dim,page,heads", [(64, 16, 3), (128, 64, 2)])
def test_read_of_ranges(B, dt, dim, page, heads):
    """Sequences of several lengths, one of them empty, from given starts; rows behind the last are left as they were."""
    s = R.Setting([33, 1, 0, 70], [5, 1, 0, 70], heads, 1, dim, page, seed=4)
    cache = tuple(t.cuda() for t in s.cache)
    starts = torch.tensor([28, 0, 0, 0], dtype=torch.int32, device="cuda")
    k, v = (torch.full((s.total + 3, heads, dim), 9.0, dtype=dt, device="cuda") for _ in range(2))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.nvfp4_kv_read(cache, s.table.cuda(), starts, s.offsets.cuda(), k, v, status)
    for part, got in enumerate((k, v)):
        pool = R.values(s.cache, part)
        want = torch.cat([R.tokens_of(pool, s.table[b], n)[:, n - m:].transpose(0, 1) for b, (n, m) in enumerate(zip(s.lens, s.queries))])
        # q s is exact, q s S rounded to fp32 once: so is the product of float64 to float32
        assert torch.equal(got[:s.total].cpu(), want.float().to(dt))
        assert (got[s.total:] == 9.0).all()
    assert status.item() == 0


def test_bounds(B):
    """Slots past the pool, tokens past the table and pages outside the pool: skipped or zero, status bit 2."""
    cache = empty_cache(2, 1, 16, 64)
    k, v = tensors(3, 1, 64, torch.bfloat16)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.nvfp4_kv_write(cache, k, v, torch.tensor([32, -5, 2 ** 40], device="cuda"), status=status)
    assert status.item() == 4 and (cache[0] == 0x55).all() and (cache[1] == 0x55).all()
    for table, start in (([[0, 2]], 14), ([[0, -1]], 14), ([[0, 1]], 30), ([[0, 1]], -2)):
        status.zero_()
        out = torch.full((4, 1, 64), 9.0, device="cuda")
        B.nvfp4_kv_read(cache, torch.tensor(table, dtype=torch.int32, device="cuda"), torch.tensor([start], dtype=torch.int32, device="cuda"),
                        torch.tensor([0, 4], dtype=torch.int32, device="cuda"), out, None, status)
        zero = out[2:] if start > 0 else out[:2]
        assert status.item() == 4 and (zero == 0).all() and (out != 9.0).all()


@pytest.mark.parametrize("method", [0, 1])
def test_not_finite(B, method):
    cache = empty_cache(1, 1, 16, 64)
    k, v = tensors(4, 1, 64, torch.float32)
    k[1, 0, 17], v[2, 0, 0], k[3] = float("nan"), float("inf"), 0.0
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.nvfp4_kv_write(cache, k, v, torch.arange(4, device="cuda"), method, status)
    assert status.item() == 1
    for part, x in enumerate((k, v)):
        codes, sf = quantised(B, x, cache[2 + part], method == B.NVFP4_KV_SWEEP)
        assert torch.equal(cache[0][0, :, part, :4].transpose(0, 1), codes)
        assert torch.equal(cache[1][0, :, part, :, :4].permute(2, 0, 1), sf)


def test_graph(B):
    cache = empty_cache(4, 2, 16, 128)
    k, v = tensors(16, 2, 128, torch.bfloat16)
    slots = torch.arange(16, device="cuda")
    out = torch.empty(16, 2, 128, device="cuda")
    table, offsets = torch.tensor([[0, 1, 2, 3]], dtype=torch.int32, device="cuda"), torch.tensor([0, 16], dtype=torch.int32, device="cuda")
    starts = torch.zeros(1, dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.nvfp4_kv_write(cache, k, v, slots)
        B.nvfp4_kv_read(cache, table, starts, offsets, out)
    for first in (3, 40):
        k.copy_(tensors(16, 2, 128, torch.bfloat16, seed=first)[0])
        slots.copy_(torch.arange(16) + first)
        starts.fill_(first)
        graph.replay()
        codes, sf = quantised(B, k, cache[2], True)
        want = torch.empty(16 * 2, 128, device="cuda")
        B.nvfp4_dequantize(codes.view(32, 64), sf.view(32, 8), B.NVFP4_SF_LINEAR, cache[2], 32, 128, 16, want)
        assert torch.equal(out.view(32, 128), want)
