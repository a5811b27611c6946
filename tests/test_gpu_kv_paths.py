"""Every path of attention over the cache -- few and many rows, parts alone, in clusters and through the workspace, with and
without a prefix -- against 64 bits, at shapes that test_kv_plans.py shows to take them."""
import math
import time

import pytest
import torch

import kv_reference as R

pytestmark = pytest.mark.gpu

# (lens, queries, heads, group, dim, page), further arguments -> rows of a block, how parts are joined, rows of the prefix's blocks
PATHS = [
    ((([100, 7], [1, 1], 2, 4, 64, 16), {}), (8, "alone", 0)),
    ((([260, 7], [1, 1], 2, 4, 128, 16), {}), (8, "cluster", 0)),
    ((([1100, 700], [2, 1], 1, 4, 64, 16), {}), (8, "cluster", 0)),
    ((([1900, 64, 1], [1, 1, 1], 2, 8, 128, 64), {}), (8, "cluster", 0)),
    ((([5000], [1], 2, 4, 128, 64), {}), (8, "workspace", 0)),
    ((([100, 128], [2, 1], 2, 8, 128, 16), {}), (16, "alone", 0)),
    ((([900, 70], [3, 2], 2, 4, 128, 16), {}), (16, "cluster", 0)),
    ((([4000], [2], 1, 7, 64, 32), {}), (16, "workspace", 0)),
    ((([40, 90], [30, 20], 38, 3, 64, 16), {}), (256, "alone", 0)),
    ((([40, 90], [30, 20], 76, 2, 128, 16), {}), (256, "alone", 0)),
    ((([700], [200], 1, 3, 128, 16), {}), (256, "workspace", 0)),
    ((([300, 1000], [6, 9], 2, 4, 64, 16), {}), (256, "workspace", 0)),
    ((([30], [1], 1, 4, 64, 16), {"prefix": 500}), (8, "merge", 8)),
    ((([30, 300], [1, 1], 1, 8, 128, 16), {"prefix": 500}), (8, "merge", 16)),
    ((([30, 9, 40], [1, 1, 1], 2, 8, 128, 16), {"prefix": 2000}), (8, "merge", 256)),
    ((([30], [2], 1, 5, 128, 16), {"prefix": 300}), (16, "merge", 16)),
    ((([30, 600], [2, 3], 2, 5, 64, 16), {"prefix": 900}), (16, "merge", 256)),
    ((([9], [1], 1, 2, 128, 16), {"prefix": 64}), (8, "merge", 8)),
    ((([50, 64], [9, 12], 2, 4, 128, 16), {"prefix": 333}), (256, "workspace", 256)),
    ((([190, 2100], [165, 170], 39, 3, 128, 32), {}), (512, "alone", 0)),
    ((([0, 2100, 160], [165, 170, 169], 26, 3, 128, 32), {}), (512, "alone", 0)),
    ((([4100], [250], 38, 2, 128, 128), {}), (512, "workspace", 0)),
    ((([3, 9, 1] * 20, [1] * 60, 10, 8, 128, 16), {"prefix": 15000}), (8, "merge", 512)),
    ((([500, 2180], [150, 170], 38, 3, 128, 64), {"prefix": 2100}), (512, "workspace", 512)),
]

@pytest.fixture(scope="module")
def B():
    from paper_2606_07618_gb300 import binding
    binding.lib()
    return binding


@pytest.mark.parametrize("args,path", PATHS, ids=[f"{i}-{p[0]}-{p[1]}-{p[2]}" for i, (_, p) in enumerate(PATHS)])
@pytest.mark.parametrize("causal", [True, False])
def test_paths(B, args, path, causal):
    s = R.Setting(*args[0], **args[1], seed=7)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out, lse = s.run(B, causal, extra=3, status=status)
    R.check(out[:s.total], s.want(causal), lse[:s.total])
    assert (out[s.total:] == 7.0).all() and status.item() == 0


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("queries", [[33, 64], [129, 1], [128], [43], [300, 90], [137, 1], [171, 170], [342], [1, 400, 341]])
def test_one_and_two_tiles_of_rows(B, dim, queries):
    """One tile's keys in two streams, two tiles, and a last tile alone, over odd numbers of key tiles."""
    for extra in (0, 100, 400):
        s = R.Setting([n + extra for n in queries], queries, 1, 3, dim, 32, seed=extra)
        out, lse = s.run(B)
        R.check(out, s.want(), lse)


def test_prefix_alone(B):
    """Sequences without tokens of their own, and a prefix of no tokens."""
    s = R.Setting([0, 0], [1, 1], 2, 4, 128, 16, seed=3, prefix=700)
    out, lse = s.run(B, causal=False)
    R.check(out, s.want(False), lse)
    for shape in (([30, 5], [1, 1], 2, 4, 128, 16), ([40, 50], [30, 20], 1, 4, 64, 16)):
        s = R.Setting(*shape, seed=4, prefix=200)
        dev = [t.cuda() for t in s.cache]
        q, out = s.q.cuda(), torch.empty_like(s.q, device="cuda")
        table, lens, offsets = s.table.cuda(), torch.tensor(s.lens, dtype=torch.int32, device="cuda"), s.offsets.cuda()
        n = max(s.queries)
        ws = torch.full((B.nvfp4_kv_attention_workspace(dev, q, 2, table.shape[1], n, s.common.numel()),), 255, dtype=torch.uint8, device="cuda")
        B.nvfp4_kv_attention_prefix(q, dev, s.common.cuda(), torch.zeros(1, dtype=torch.int32, device="cuda"), table, lens, offsets, n,
                                    s.scale, out, workspace=ws)
        s.prefix = 0
        s.common = s.common[:0]
        R.check(out, s.want())


@pytest.mark.parametrize("queries", [1, 40])
def test_a_prefix_of_no_pages(B, queries):
    """No prefix at all, by the call that takes one."""
    s = R.Setting([300, 50], [queries, 1], 2, 4, 128, 16, seed=4)
    want = s.run(B)
    cache = tuple(t.cuda() for t in s.cache)
    q, table, lens, offsets = s.q.cuda(), s.table.cuda(), torch.tensor(s.lens, dtype=torch.int32, device="cuda"), s.offsets.cuda()
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    none, zero = torch.empty(0, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = torch.empty(B.nvfp4_kv_attention_workspace(cache, q, 2, table.shape[1], queries), dtype=torch.uint8, device="cuda")
    B.nvfp4_kv_attention_prefix(q, cache, none, zero, table, lens, offsets, queries, s.scale, out, True, lse, ws)
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


def test_fewer_queries_than_max_q(B):
    """max_q above the longest sequence's queries, and below it: those past it are not computed."""
    s = R.Setting([90, 40], [3, 1], 2, 4, 64, 16, seed=5)
    want = s.want()
    for n in (3, 4, 100):
        out, lse = s.run(B, max_q=n)
        R.check(out, want, lse)
    out, _ = s.run(B, max_q=2)
    assert (out[2] == 7.0).all()
    R.check(torch.cat((out[:2], out[3:])), [torch.cat((w[:2], w[3:])) for w in want])


def test_pages_shared_and_out_of_order(B):
    """Two sequences that hold the same pages, in another order each."""
    s = R.Setting([64, 64], [1, 1], 1, 4, 128, 16, seed=6)
    s.table[1] = s.table[0].flip(0)
    out, lse = s.run(B)
    R.check(out, s.want(), lse)


@pytest.mark.parametrize("shape", [([40], [1], 2, 4, 128, 16), ([40, 300], [3, 70], 2, 4, 128, 16), ([300, 40], [70, 40], 1, 3, 64, 16),
                                   ([180, 2100], [165, 170], 38, 3, 128, 32)])
@pytest.mark.parametrize("causal", [True, False])
def test_hidden_pages_and_queries_that_are_not_finite(B, shape, causal):
    """Page numbers outside the pool hide their tokens of every kernel (page 0, which none holds, is NaN); a NaN and an infinity
    stay in their rows."""
    s = R.Setting(*shape, seed=21)
    free = next(i for i in range(s.cache[0].shape[0]) if not (s.table == i).any())
    s.table[s.table == 0] = free
    for t in s.cache[:2]:
        t[free] = t[0]
    s.cache[1][0] = 0x7F
    b, n, m = len(s.lens) - 1, s.lens[-1], s.queries[-1]
    row, good = s.table[b].clone(), torch.ones(n, dtype=torch.bool)
    for i, bad in ((0, -1), (2, s.cache[0].shape[0]), ((n - 1) // s.page, 2 ** 31 - 1)):
        s.table[b, i] = bad
        good[i * s.page:(i + 1) * s.page] = False
    q, status = s.q.cuda(), torch.zeros(1, dtype=torch.int32, device="cuda")
    q[0, 1, 3], q[-1, -1, 9] = math.nan, math.inf
    out, lse = s.run(B, causal, q=q, status=status)
    assert status.item() == 4
    k, v = (R.tokens_of(R.values(s.cache, i), row, n)[:, good] for i in (0, 1))
    sees = good.long().cumsum(0)[(n - m + torch.arange(m)).clamp(min=0) if causal else torch.full((m,), n - 1)]
    assert not causal or n >= m
    last = R.attention(s.q[-m:].double().view(m, s.heads, s.group, s.dim), k, v, s.scale, sees)
    rest = R.Setting(*shape, seed=21)
    rest.table, rest.cache = s.table.clone(), s.cache
    rest.table[b] = row
    want = [torch.cat((w[:-m], x)) for w, x in zip(rest.want(causal), last)]
    nan = torch.zeros(s.total, s.heads * s.group, dtype=torch.bool)
    nan[0, 1] = nan[-1, -1] = True
    assert torch.equal(torch.isnan(out.cpu()).all(-1), nan) and torch.equal(torch.isnan(out.cpu()).any(-1), nan)
    want = [w.masked_fill(nan.view(s.total, s.heads, s.group, *[1] * (w.dim() - 3)), 0) for w in want]
    R.check(out.masked_fill(nan.cuda()[..., None], 0), want)


@pytest.mark.parametrize("queries", [1, 4, 20, 170])
def test_a_pool_past_4_gb(B, queries):
    """The same bits from pages at the end of a pool whose offsets pass 32 bits."""
    s = R.Setting([2100], [queries], 38, 3, 128, 64, seed=22)
    pages, heads = s.cache[0].shape[:2]
    total = 2 ** 33 // (heads * 64 * 128) + 7
    want = s.run(B)
    codes = torch.empty(total, *s.cache[0].shape[1:], dtype=torch.uint8, device="cuda")
    sf = torch.empty(total, *s.cache[1].shape[1:], dtype=torch.uint8, device="cuda")
    codes[-pages:], sf[-pages:] = s.cache[0].cuda(), s.cache[1].cuda()
    s.cache = (codes, sf, *s.cache[2:])
    s.table += (total - pages)
    for a, b in zip(s.run(B), want):
        assert torch.equal(a, b)
    # read back, and written again at the end
    cache = (codes, sf, *(t.cuda() for t in s.cache[2:]))
    k = torch.empty(2100, heads, 128, device="cuda")
    v = torch.empty_like(k)
    table, offsets = s.table.cuda(), torch.tensor([0, 2100], dtype=torch.int32, device="cuda")
    B.nvfp4_kv_read(cache, table, None, offsets, k, v)
    for i, x in enumerate((k, v)):
        assert torch.equal(R.tokens_of(R.values((codes[-pages:].cpu(), sf[-pages:].cpu(), *s.cache[2:]), i), s.table[0] - (total - pages), 2100)
                           .permute(1, 0, 2).float(), x.cpu())
    slots = (s.table[0].long().repeat_interleave(64) * 64 + torch.arange(64).repeat(s.table.shape[1]))[:2100].cuda()
    B.nvfp4_kv_write(cache, k, v, slots, B.NVFP4_KV_ABSMAX)
    small = tuple(torch.zeros(pages, *t.shape[1:], dtype=torch.uint8, device="cuda") for t in (codes, sf)) + cache[2:]
    B.nvfp4_kv_write(small, k, v, slots - (total - pages) * 64, B.NVFP4_KV_ABSMAX)
    used = torch.zeros(pages * 64, dtype=torch.bool, device="cuda")
    used[slots - (total - pages) * 64] = True
    used = used.view(pages, 64)
    for a, b, at in ((codes, small[0], 3), (sf, small[1], 4)):
        a = a[-pages:].movedim(at, 1)[used]
        assert torch.equal(a, b.movedim(at, 1)[used])


def test_streams(B):
    """Two calls at one time on two streams, each with a workspace of its own."""
    sets = [R.Setting([3000 + i, 50], [1, 1], 2, 4, 128, 16, seed=i, prefix=600 * i) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in sets]
    outs = []
    torch.cuda.synchronize()
    for s, stream in zip(sets, streams):
        with torch.cuda.stream(stream):
            outs.append(s.run(B))
    torch.cuda.synchronize()
    for s, (out, lse) in zip(sets, outs):
        R.check(out, s.want(), lse)


def test_two_graphs_share_a_workspace(B):
    s = R.Setting([900, 80], [1, 1], 2, 4, 128, 16, seed=9, prefix=500)
    t = R.Setting([4100], [1], 2, 4, 128, 16, seed=10)
    calls, graphs = [], []
    ws = None
    for x in (s, t):
        dev = [c.cuda() for c in x.cache]
        q, out = x.q.cuda(), torch.empty_like(x.q, device="cuda")
        table, lens, offsets = x.table.cuda(), torch.tensor(x.lens, dtype=torch.int32, device="cuda"), x.offsets.cuda()
        common, plen = x.common.cuda(), torch.tensor([x.prefix], dtype=torch.int32, device="cuda")
        need = B.nvfp4_kv_attention_workspace(dev, q, len(x.lens), table.shape[1], 1, common.numel())
        calls.append((dev, q, out, table, lens, offsets, common, plen, need))
    ws = torch.full((max(c[-1] for c in calls),), 255, dtype=torch.uint8, device="cuda")
    for x, (dev, q, out, table, lens, offsets, common, plen, _) in zip((s, t), calls):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            if x.prefix:
                B.nvfp4_kv_attention_prefix(q, dev, common, plen, table, lens, offsets, 1, x.scale, out, workspace=ws)
            else:
                B.nvfp4_kv_attention(q, dev, table, lens, offsets, 1, x.scale, out, workspace=ws)
        graphs.append(g)
    for _ in range(20):
        for g in graphs:
            g.replay()
    for x, c in zip((s, t), calls):
        R.check(c[2], x.want())


@pytest.mark.parametrize("shape", [([40, 90], [30, 20], 38, 3, 64, 16), ([190, 2100], [165, 170], 39, 3, 128, 32)])
def test_wait_runs_out_and_is_reported(B, shape):
    """The waits for keys give up after their limit (of single blocks and of pairs), nothing is written, and the context stays usable."""
    s = R.Setting(*shape, seed=11)
    n = max(s.queries)
    dev = [t.cuda() for t in s.cache]
    q, out = s.q.cuda(), torch.full_like(s.q, 7.0, device="cuda")
    table, lens, offsets = s.table.cuda(), torch.tensor(s.lens, dtype=torch.int32, device="cuda"), s.offsets.cuda()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    assert B.nvfp4_kv_attention_workspace(dev, q, 2, table.shape[1], n) == 0
    torch.cuda.synchronize()
    t0 = time.time()
    B.nvfp4_kv_selftest_wait_timeout(q, dev, table, lens, offsets, n, s.scale, out, status)
    torch.cuda.synchronize()
    assert 0.5 < time.time() - t0 < 60
    assert status.item() == 16 and (out == 7.0).all()
    out, lse = s.run(B)
    R.check(out, s.want(), lse)
