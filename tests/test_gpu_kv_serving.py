"""The cache's operators together, as a serving program uses them: prompts, decoding steps, drafted tokens and shared prompts
over several layers, against attention in 64 bits over the values that the cache holds."""
import pytest
import torch

import kv_reference as R

pytestmark = pytest.mark.gpu
HEADS, GROUP = 2, 4


@pytest.fixture(scope="module")
def K():
    from paper_2606_07618_gb300 import kv_cache
    return kv_cache


def draw(n, heads, dim, g):
    return torch.randn(n, heads, dim, generator=g).to(torch.bfloat16).cuda()


def want_of(cache, pages, seqs, counts, q, scale):
    """attention() of kv_reference for a step's queries, from the books of the pages."""
    held = tuple(t.cpu() for t in cache.held)
    pools = [R.values(held, part) for part in (0, 1)]
    rows, at = [], 0
    for seq, n in zip(seqs, counts):
        s = pages.sequences[seq]
        k, v = (R.tokens_of(p, torch.tensor(s.pages), s.length) for p in pools)
        before = 0
        if s.prefix:
            before = s.prefix.length
            k, v = (torch.cat((R.tokens_of(p, torch.tensor(s.prefix.pages), before), x), 1) for p, x in zip(pools, (k, v)))
        x = q[at:at + n].cpu().double().view(n, HEADS, GROUP, cache.dim)
        rows.append(R.attention(x, k, v, scale, before + s.length - n + 1 + torch.arange(n)))
        at += n
    return [torch.cat([r[i] for r in rows]) for i in range(5)]


@pytest.mark.parametrize("dim,page", [(64, 16), (128, 64)])
def test_serving(K, dim, page):
    g = torch.Generator().manual_seed(dim)
    pages, rotary = K.Pages(120, page), K.Rotary(dim, 10000.0)
    sample = draw(100, HEADS, dim, g)
    S = K.KVCache.calibrate(sample * 2)
    caches = [K.KVCache(pages, HEADS, dim, S, S) for _ in range(2)]
    kept = {}                                                      # what was written, turned: (layer, sequence) -> keys, values

    def forward(counts):
        step = pages.step(list(counts.items()))
        seqs, ns = list(counts), list(counts.values())
        for i, cache in enumerate(caches):
            qkv = draw(step.tokens, HEADS * (GROUP + 2), dim, g)   # a projection's columns: queries, keys, values
            q, k, v = qkv[:, :HEADS * GROUP], qkv[:, HEADS * GROUP:HEADS * (GROUP + 1)], qkv[:, HEADS * (GROUP + 1):]
            plain = qkv[:, :HEADS * (GROUP + 1)].clone()
            rotary(qkv[:, :HEADS * (GROUP + 1)], step.positions)   # queries and keys at once
            turned = R.rope(plain.cpu(), step.positions.cpu(), rotary.turns.cpu().double() * (2 * torch.pi / 2.0 ** 64), 1.0, True, False)
            assert ((qkv[:, :HEADS * (GROUP + 1)].cpu().double() - turned).abs() <= 2.0 ** -8 * turned.abs() + 2.0 ** -18).all()
            cache.write(step, k, v)
            out = cache.attend(step, q)
            R.check(out, want_of(cache, pages, seqs, ns, q, dim ** -0.5))
            at = 0
            for seq, n in zip(seqs, ns):
                kept.setdefault((i, seq), []).append((k[at:at + n].clone(), v[at:at + n].clone()))
                at += n
        return step

    a, b, c = pages.add(), pages.add(), pages.add()
    forward({a: 70, b: 1, c: 33})                                  # prompts
    for _ in range(3):
        forward({c: 1, a: 1, b: 1})                                # decoding, in another order
    forward({b: 4, a: 3})                                          # drafted tokens; c waits
    pages.drop(c)
    d = pages.add()
    forward({d: 50, a: 1})                                         # on pages that c left
    pre = pages.share(b)
    e, f = pages.add(pre), pages.add(pre)
    forward({e: 5, f: 1})
    forward({f: 1, e: 1})
    for i, cache in enumerate(caches):
        assert cache.status.item() == 0
        for seq in (a, d, e, f):
            got = cache.read(seq, torch.float32)
            for part in (0, 1):
                x = torch.cat([w[part] for w in kept[i, seq]])
                # an element is off by at most the block's largest over 6 (the top step of E2M1) and an eighth of itself (E4M3 scale)
                tol = (x.float().view(*x.shape[:2], -1, 16).abs().amax(-1, keepdim=True) / 4).expand(*x.shape[:2], -1, 16).reshape(x.shape)
                assert ((got[part] - x.float()).abs() <= tol + float(S)).all()


def test_a_step_in_a_graph(K):
    """One decoding step captured and replayed with new tokens: the same as eager calls."""
    g = torch.Generator().manual_seed(1)
    pages, rotary = K.Pages(40, 16), K.Rotary(64, 10000.0)
    caches = [K.KVCache(pages, HEADS, 64, 0.01, 0.01) for _ in range(2)]
    a, b = pages.add(), pages.add()
    step = pages.step([(a, 40), (b, 17)])
    first = [draw(step.tokens, HEADS, 64, g) for _ in range(2)]
    for c in caches:
        c.write(step, *first)
    step = pages.step([(a, 1), (b, 1)])
    q, k, v = draw(2, HEADS * GROUP, 64, g), draw(2, HEADS, 64, g), draw(2, HEADS, 64, g)
    q0, k0 = q.clone(), k.clone()

    def forward(cache):
        rotary(k0, step.positions, k)
        rotary(q0, step.positions, q)
        cache.write(step, k, v)
        return cache.attend(step, q)
    want = forward(caches[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = forward(caches[0])
    for _ in range(2):
        graph.replay()
    assert torch.equal(out, want)
    for t in (q0, k0, v):
        t.copy_(torch.randn(t.shape, generator=g).to(t.dtype))
    graph.replay()
    got = out.clone()
    assert torch.equal(got, forward(caches[1]))


def test_demonstration_runs(K, capsys):
    K.main(batch=2, length=100)
    assert "relative error" in capsys.readouterr().out
