"""Plain 64-bit forms of the key/value cache's operators, and caches and tables to try them on (torch on the CPU)."""
import math

import torch

E2M1 = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


def e4m3(codes):
    c = codes.long()
    e, m = (c >> 3) & 15, (c & 7).double()
    v = torch.where(e == 0, m * 2.0 ** -9, (1 + m / 8) * torch.pow(2.0, (e - 7).double()))
    return torch.where((c & 127) == 127, torch.full_like(v, math.nan), v)


def values(cache, part):
    """Keys (part 0) or values (1) of the whole pool: [pages, heads, page, dim] float64."""
    codes, sf = cache[0].cpu()[:, :, part], cache[1].cpu()[:, :, part]
    S = cache[2 + part].cpu().double()
    q = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).long()
    x = torch.where(q >= 8, -E2M1[q & 7], E2M1[q & 7])
    return x * e4m3(sf).transpose(-1, -2).repeat_interleave(16, -1) * S


def tokens_of(pool, row, n):
    """The first n tokens of the pages in row: [heads, n, dim]."""
    page = pool.shape[2]
    ids = row[:-(-n // page)].long()
    return pool[ids].permute(1, 0, 2, 3).flatten(1, 2)[:, :n]


def attention(q, k, v, scale, past):
    """q [n, heads, group, dim], k, v [heads, keys, dim], query i sees keys below past[i].  Returns out, lse, the sum of weighted
    magnitudes (what the weights' rounding errors scale with), a bound on the logits' fp32 error and the sum of magnitudes."""
    n, heads, group, dim = q.shape
    z = torch.einsum("nhgd,hkd->nhgk", q, k) * scale
    keys = torch.arange(k.shape[1])
    hide = keys[None, :] >= past[:, None]
    z = z.masked_fill(hide[:, None, None], -math.inf)
    out, lse = torch.zeros(n, heads, group, dim, dtype=torch.float64), torch.full((n, heads, group), -math.inf, dtype=torch.float64)
    mag, off, total = torch.zeros_like(out), torch.zeros_like(lse), torch.zeros_like(out)
    for i in range(n):
        m = int(min(max(past[i], 0), k.shape[1]))
        if m == 0:
            continue
        p = torch.softmax(z[i, :, :, :m], -1)
        out[i] = torch.einsum("hgk,hkd->hgd", p, v[:, :m])
        mag[i] = torch.einsum("hgk,hkd->hgd", p, v[:, :m].abs())
        total[i] = v[:, :m].abs().sum(1)[:, None]
        lse[i] = torch.logsumexp(z[i, :, :, :m], -1)
        size = torch.einsum("hgd,hkd->hgk", q[i].abs(), k[:, :m].abs()).amax(-1)
        top = q[i].abs().amax(-1) * k[:, :m].abs().sum(-1).amax(-1)[:, None]
        # a sum of dim products in fp32, the factor's roundings; the queries' smallest elements
        off[i] = scale * ((dim + 8) * 2.0 ** -24 * size + 2.0 ** -25 * top)
    return out, lse, mag, off, total


def check(got, want, lse=None):
    """got (bf16) and lse (fp32) of attention() against its results: a weight is off by 2^-11 (fp16), by its logit's error, which
    the sum of weights has too, and by a few roundings of fp32; the result by half a step of bf16.  fp16's last bit is
    2^-24, and weights are held so that the largest is at least 2^7: however small, each is off by up to 2^-25 2^-7 = 2^-32 of the
    largest, which is at most the sum that divides (an element whose larger weights all meet zeros shows it)."""
    out, ref_lse, mag, off, total = want
    got = got.double().cpu().view(out.shape)
    tol = 2.0 ** -8 * out.abs() + (2.0 ** -11 + 2 * off + 2.0 ** -18)[..., None] * mag * 1.01 + 2.0 ** -32 * total
    bad = ~((got - out).abs() <= tol)
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} off, most {((got - out).abs() / tol.clamp(min=1e-300)).max():.3g} of the tolerance"
    if lse is not None:
        g = lse.double().cpu().view(ref_lse.shape)
        empty = torch.isinf(ref_lse)
        assert torch.equal(empty, g == -math.inf)
        d = (g - ref_lse).abs()[~empty]
        assert (d <= (2.0 ** -18 + off + 2.0 ** -22 * ref_lse.abs())[~empty]).all(), d.max()


class Setting:
    """A batch of sequences with random pages of a random cache (CPU; to(device) for the calls)."""

    def __init__(self, lens, queries, heads, group, dim, page, seed=0, prefix=0, spare=3, spread=1.0):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.queries, self.prefix = lens, queries, prefix
        self.heads, self.group, self.dim, self.page = heads, group, dim, page
        counts = [-(-n // page) for n in lens]
        common = -(-prefix // page)
        pages = sum(counts) + common + spare
        ids = torch.randperm(pages, generator=g).int()
        self.common, ids = ids[:common], ids[common:]
        width = max(counts + [1])
        self.table = torch.full((len(lens), width), -7, dtype=torch.int32)
        at = 0
        for b, n in enumerate(counts):
            self.table[b, :n] = ids[at:at + n]
            at += n
        codes = torch.randint(0, 256, (pages, heads, 2, page, dim // 2), generator=g).to(torch.uint8)
        sf = torch.randint(0x20, 0x48, (pages, heads, 2, dim // 16, page), generator=g).to(torch.uint8)
        # what no sequence holds: NaN scales
        used = torch.zeros(pages, page, dtype=torch.bool)
        for row, n in [(self.table[b], n) for b, n in enumerate(lens)] + [(self.common, prefix)]:
            for j in range(n):
                used[int(row[j // page]), j % page] = True
        sf.permute(0, 4, 1, 2, 3)[~used] = 0x7F
        self.cache = (codes, sf, torch.tensor([0.11]), torch.tensor([0.37]))
        self.offsets = torch.zeros(len(lens) + 1, dtype=torch.int32)
        self.offsets[1:] = torch.tensor(queries).cumsum(0)
        self.total = int(self.offsets[-1])
        scale = torch.exp(spread * torch.randn(self.total, heads * group, 1, generator=g))
        self.q = (torch.randn(self.total, heads * group, dim, generator=g) * scale).to(torch.bfloat16)
        self.scale = dim ** -0.5

    def want(self, causal=True):
        """attention() of all rows, sequence after sequence."""
        pools = [values(self.cache, part) for part in (0, 1)]
        pre = [tokens_of(p, self.common, self.prefix) for p in pools]
        rows = []
        for b, (n, m) in enumerate(zip(self.lens, self.queries)):
            k, v = (torch.cat((x, tokens_of(p, self.table[b], n)), 1) for p, x in zip(pools, pre))
            q = self.q[self.offsets[b]:self.offsets[b + 1]].double().view(m, self.heads, self.group, self.dim)
            own = n - m + 1 + torch.arange(m) if causal else torch.full((m,), n)
            rows.append(attention(q, k, v, self.scale, self.prefix + own.clamp(min=0)))
        return [torch.cat([r[i] for r in rows]) for i in range(5)]

    def run(self, B, causal=True, out=None, lse=None, extra=0, status=None, max_q=None, q=None):
        """The call on the GPU: out [total + extra, heads * group, dim], and lse."""
        dev = "cuda"
        cache = tuple(t.to(dev) for t in self.cache)
        q = self.q.to(dev) if q is None else q
        if extra:
            q = torch.cat((q, torch.ones(extra, *q.shape[1:], dtype=q.dtype, device=dev)))
        out = torch.full_like(q, 7.0, memory_format=torch.contiguous_format) if out is None else out
        lse = torch.full(q.shape[:2], 7.0, device=dev) if lse is None else lse
        table, lens, offsets = self.table.to(dev), torch.tensor(self.lens, dtype=torch.int32, device=dev), self.offsets.to(dev)
        max_q = max(self.queries) if max_q is None else max_q
        args = (table, lens, offsets, max_q, self.scale, out, causal, lse)
        n = self.common.numel()
        ws = torch.full((B.nvfp4_kv_attention_workspace(cache, q, len(self.lens), table.shape[1], max_q, n),), 255,
                        dtype=torch.uint8, device=dev)
        if self.prefix:
            B.nvfp4_kv_attention_prefix(q, cache, self.common.to(dev), torch.tensor([self.prefix], dtype=torch.int32, device=dev),
                                        *args, workspace=ws, status=status)
        else:
            B.nvfp4_kv_attention(q, cache, *args, workspace=ws, status=status)
        return out, lse


def rope(x, positions, freqs, magnitude, halves, inverse):
    """Rotary positions in 64 bits: freqs in radians a position."""
    x = x.double()
    half = freqs.numel()
    t = positions.double()[:, None] * freqs.double()[None, :] * (-1 if inverse else 1)
    c, s = (magnitude * f(t)[:, None, :] for f in (torch.cos, torch.sin))
    y = x.clone()
    i = torch.arange(half)
    a, b = (i, i + half) if halves else (2 * i, 2 * i + 1)
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., a] * s + x[..., b] * c
    return y
