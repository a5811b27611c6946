"""Attention over the NVFP4 cache, also behind a shared prefix, against 64 bits: lengths, heads, pages, masks, strides."""
import math

import pytest
import torch

import kv_reference as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2606_07618_gb300 import binding
    binding.lib()
    return binding


def run(B, s, causal=True):
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out, lse = s.run(B, causal, extra=2, status=status)
    R.check(out[:s.total], s.want(causal), lse[:s.total])
    assert (out[s.total:] == 7.0).all() and (lse[s.total:] == 7.0).all()       # rows behind the last sequence
    assert status.item() == 0


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads,group", [(1, 1), (2, 3), (1, 8), (3, 4), (1, 9), (2, 16), (1, 40)])
def test_single_tokens(B, dim, heads, group):
    run(B, R.Setting([1, 2, 15, 16, 17, 63, 64, 65, 200, 333], [1] * 10, heads, group, dim, 16, seed=group))


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 1024])
def test_pages(B, dim, page):
    run(B, R.Setting([1, page - 1, page, page + 1, 300], [1, 2, 1, 1, 3], 2, 2, dim, page, seed=page))


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("group", [1, 4, 7])
def test_chunks(B, dim, causal, group):
    """Several queries a sequence, more than one tile of rows, whole prompts, and sequences without queries or without tokens."""
    run(B, R.Setting([50, 130, 7, 0, 40, 400], [50, 33, 0, 0, 1, 129], 2, group, dim, 32, seed=group), causal)


@pytest.mark.parametrize("dim", [64, 128])
def test_queries_that_see_nothing(B, dim):
    """More queries than cached tokens: the first ones see none (causal)."""
    run(B, R.Setting([3, 0, 1, 20], [5, 2, 40, 21], 1, 2, dim, 16, seed=8))


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("b,new", [(1, 1), (3, 2), (9, 4), (40, 1), (2, 70)])
def test_prefix(B, dim, b, new):
    lens = [new + 7 * i for i in range(b)]
    run(B, R.Setting(lens, [new] * b, 2, 3, dim, 16, seed=b, prefix=211))


@pytest.mark.parametrize("prefix", [1, 16, 64, 1000, 4097])
def test_prefix_lengths(B, prefix):
    run(B, R.Setting([1, 0, 30, 5], [1, 0, 2, 7], 1, 4, 128, 32, seed=prefix, prefix=prefix), causal=prefix != 64)


def test_long(B):
    """Long enough for many parts."""
    run(B, R.Setting([9001, 12], [1, 1], 1, 4, 128, 64, seed=5))
    run(B, R.Setting([20000], [3], 1, 2, 64, 128, seed=6))


def test_heavy_logits(B):
    """Queries of large and small sizes: weights that are almost one, and almost equal."""
    for spread in (3.0, 6.0):
        s = R.Setting([700, 90], [2, 4], 2, 2, 128, 16, seed=11, spread=spread)
        out, lse = s.run(B)
        want = s.want()
        R.check(out, want, lse)


def test_zero_scale_is_the_mean(B):
    s = R.Setting([37, 100], [1, 3], 1, 2, 64, 16, seed=12)
    s.scale = 0.0
    run(B, s)


def test_query_sizes(B):
    """Rows of zeros, of the smallest and of large numbers."""
    s = R.Setting([45, 45, 45], [1, 1, 1], 1, 2, 64, 16, seed=13)
    s.q[0] = 0
    s.q[1] *= 2.0 ** -120
    s.scale = 2.0 ** -3
    s.q[2, 0] *= 2.0 ** 5
    run(B, s)


def test_queries_that_are_not_finite(B):
    """NaN and infinities in a query stay in its row."""
    s = R.Setting([30, 70], [2, 1], 1, 4, 128, 16, seed=14)
    q = s.q.cuda()
    q[0, 1, 3], q[2, 2, 9] = math.nan, math.inf
    out, lse = s.run(B, q=q)
    bad = torch.zeros(3, 4, dtype=torch.bool)
    bad[0, 1] = bad[2, 2] = True
    assert torch.equal(torch.isnan(out.cpu()).all(-1), bad) and torch.equal(torch.isnan(out.cpu()).any(-1), bad)
    assert torch.equal(torch.isnan(lse.cpu()), bad)
    want = [w.masked_fill(bad.view(3, 1, 4, *[1] * (w.dim() - 3)), 0) for w in s.want()]
    R.check(out.masked_fill(bad.cuda()[..., None], 0), want)


@pytest.mark.parametrize("first,pad", [(0, 0), (8, 0), (1, 0), (0, 1)])
def test_strides(B, first, pad):
    """q and out as columns of one buffer, at any alignment."""
    s = R.Setting([50, 70], [1, 3], 2, 2, 64, 16, seed=15)
    heads = s.heads * s.group
    plain, _ = s.run(B)
    buf = torch.full((s.total, 2 * heads * 64 + first + pad), 3.0, dtype=torch.bfloat16, device="cuda")
    q, out = (buf[:, first + i * heads * 64:first + (i + 1) * heads * 64].unflatten(1, (heads, 64)) for i in (0, 1))
    q.copy_(s.q)
    s.run(B, q=q, out=out)
    assert torch.equal(out, plain) and torch.equal(q.cpu(), s.q)
    q, out = (torch.empty(heads, s.total, 64, dtype=torch.bfloat16, device="cuda").transpose(0, 1) for _ in range(2))
    q.copy_(s.q)
    s.run(B, q=q, out=out)
    assert torch.equal(out, plain)


def test_bad_pages_and_lengths(B):
    """Page numbers outside the pool hide their tokens, lengths past the table count as the table's: status bit 2."""
    s = R.Setting([64], [1], 1, 2, 64, 16, seed=16)
    row = s.table[0].clone()
    for bad in (-1, s.cache[0].shape[0], 2 ** 31 - 1):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        s.table[0, 1] = bad
        out, lse = s.run(B, status=status)
        pools = [R.values(s.cache, i) for i in (0, 1)]
        seen = torch.cat((torch.arange(16), torch.arange(32, 64)))
        k, v = (p[row.long()].permute(1, 0, 2, 3).flatten(1, 2)[:, seen] for p in pools)
        R.check(out, R.attention(s.q.double().view(1, 1, 2, 64), k, v, s.scale, torch.tensor([48])), lse)
        assert status.item() == 4
    s.table[0] = row
    want = s.want()
    for n in (65, 2 ** 31 - 1):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        s.lens = [n]
        out, lse = s.run(B, status=status)
        R.check(out, want, lse)
        assert status.item() == 4
    s.lens = [-3]
    out, lse = s.run(B)
    assert (out == 0).all() and (lse == -math.inf).all()


def test_offsets_outside(B):
    """Offsets that leave q: the sequence is not computed, nothing else is touched, status bit 2."""
    s = R.Setting([40, 40], [1, 1], 1, 2, 64, 16, seed=17)
    s.offsets = torch.tensor([0, 1, 2 ** 30], dtype=torch.int32)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out, lse = s.run(B, status=status)
    assert status.item() == 4 and (out[1] == 7.0).all() and (out[0] != 7.0).all()


@pytest.mark.parametrize("prefix", [0, 600])
def test_graph(B, prefix):
    """Captured once, replayed for other lengths, pages and queries."""
    s = R.Setting([300, 45], [1, 1], 2, 4, 128, 16, seed=18, prefix=prefix)
    dev = [t.cuda() for t in s.cache]
    q, out = s.q.cuda(), torch.empty_like(s.q, device="cuda")
    table, lens, offsets = s.table.cuda(), torch.tensor(s.lens, dtype=torch.int32, device="cuda"), s.offsets.cuda()
    common, plen = s.common.cuda(), torch.tensor([prefix], dtype=torch.int32, device="cuda")
    ws = torch.empty(B.nvfp4_kv_attention_workspace(dev, q, 2, table.shape[1], 1, common.numel()), dtype=torch.uint8, device="cuda")

    def call():
        if prefix:
            B.nvfp4_kv_attention_prefix(q, dev, common, plen, table, lens, offsets, 1, s.scale, out, workspace=ws)
        else:
            B.nvfp4_kv_attention(q, dev, table, lens, offsets, 1, s.scale, out, workspace=ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    graph.replay()
    R.check(out, s.want())
    s.lens, s.q = [17, 40], s.q.flip(0)
    lens.copy_(torch.tensor(s.lens))
    q.copy_(s.q)
    if prefix:
        s.prefix = 333
        plen.fill_(333)
    graph.replay()
    R.check(out, s.want())


def test_same_results_again(B):
    s = R.Setting([5000, 700], [1, 2], 2, 4, 128, 16, seed=19, prefix=900)
    first = s.run(B)[0]
    for _ in range(3):
        assert torch.equal(s.run(B)[0], first)
