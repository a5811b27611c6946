"""The operators on a key/value cache in NVFP4 whose speed is measured, with their plain forms.

The cache is a pool of pages: codes [pages, heads, 2, page, dim/2] (packed E2M1; K, then V), E4M3 scales of blocks of 16
along dim, sf [pages, heads, 2, dim/16, page], and one fp32 scale for all keys and one for all values.  Sequence b's
token j lies in page table[b, j // page] at j % page.  Each case is one pass of a serving or tuning program:

  rope    rotary positions of the query and key heads of a projection's output, or (inverse) its gradient
  cache   new tokens' keys and values into the cache as 4-bit blocks, and the same tokens read back
  attend  attention of each sequence's newest tokens over its cached ones, causal
  prefix  the same for a batch whose sequences share a long prefix besides their own tokens

Values are the repository's synthetic K, V and Q: N(0, 1) with a factor exp(0.5 N(0, 1)) for each head.
"""
import math

import torch

own = False

E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # a decode batch of 16 tokens: 32 query and 8 key heads side by side, as a projection leaves them (the smallest call)
        {"name": "rope_decode", "kind": "rope", "t": 16, "heads": 40, "dim": 128, "rot": 128, "dt": "bf16", "pairs": "half",
         "inverse": False, "factor": 1.0, "far": 131072},
        # a prompt of 8192 tokens with frequencies stretched for long contexts
        {"name": "rope_prompt", "kind": "rope", "t": 8192, "heads": 40, "dim": 128, "rot": 128, "dt": "bf16", "pairs": "half",
         "inverse": False, "factor": 8.0, "far": 131072},
        # the gradient in fp32, three quarters of each head rotated in neighbouring pairs
        {"name": "rope_grad", "kind": "rope", "t": 1777, "heads": 24, "dim": 64, "rot": 48, "dt": "f32", "pairs": "neighbours",
         "inverse": True, "factor": 1.0, "far": 8192},
        # one token for each of 16 sequences at their odd lengths
        {"name": "cache_decode", "kind": "cache", "b": 16, "len": 4096, "ragged": True, "new": 1, "heads": 8, "dim": 128,
         "page": 64, "dt": "bf16", "method": "sweep"},
        # the cache of 16 sequences of 4096 tokens, block scales swept
        {"name": "cache_prompt", "kind": "cache", "b": 16, "len": 4096, "ragged": False, "new": 4096, "heads": 8, "dim": 128,
         "page": 64, "dt": "bf16", "method": "sweep"},
        # fp32 keys and values of prompts of odd lengths, small pages, scales from the block maximum
        {"name": "cache_ragged", "kind": "cache", "b": 7, "len": 3001, "ragged": True, "new": 3001, "heads": 5, "dim": 64,
         "page": 16, "dt": "f32", "method": "absmax"},
        # one sequence of 1000 tokens decoding: latency
        {"name": "attend_one", "kind": "attend", "b": 1, "len": 1000, "ragged": False, "new": 1, "heads": 8, "group": 4,
         "dim": 128, "page": 64},
        # 16 sequences of 4096 tokens decoding
        {"name": "attend_decode", "kind": "attend", "b": 16, "len": 4096, "ragged": False, "new": 1, "heads": 8, "group": 4,
         "dim": 128, "page": 64},
        # a ragged batch of 37 sequences up to 20000 tokens, two drafted tokens each, small pages
        {"name": "attend_ragged", "kind": "attend", "b": 37, "len": 20000, "ragged": True, "new": 2, "heads": 4, "group": 7,
         "dim": 64, "page": 16},
        # a chunk of 2048 prompt tokens of each of two sequences, after 6144 cached ones (the most work)
        {"name": "attend_chunk", "kind": "attend", "b": 2, "len": 8192, "ragged": False, "new": 2048, "heads": 8, "group": 4,
         "dim": 128, "page": 64},
        # 64 sequences decode behind a common prompt of 32768 tokens
        {"name": "prefix_decode", "kind": "prefix", "prefix": 32768, "b": 64, "len": 500, "ragged": True, "new": 1, "heads": 8,
         "group": 4, "dim": 128, "page": 64},
        # nine candidate answers to one short prompt of odd length, four drafted tokens each, one key head
        {"name": "prefix_drafts", "kind": "prefix", "prefix": 2011, "b": 9, "len": 129, "ragged": True, "new": 4, "heads": 1,
         "group": 8, "dim": 64, "page": 16},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rope", "cache", "attend", "attend", "prefix"])
    dim = rng.choice([64, 128, 128])
    page = rng.choice([16, 32, 64, 128])
    if kind == "rope":
        return {"kind": kind, "t": _log(rng, 1, 8192), "heads": _log(rng, 1, 40), "dim": dim,
                "rot": rng.choice([dim, dim, dim // 2, dim // 4 * 3]), "dt": rng.choice(["bf16", "bf16", "f32"]),
                "pairs": rng.choice(["half", "neighbours"]), "inverse": rng.random() < 0.3,
                "factor": rng.choice([1.0, 1.0, 4.0, 8.0]), "far": _log(rng, 8192, 1000000)}
    heads = rng.choice([1, 2, 4, 5, 8])
    if kind == "cache":
        length = _log(rng, 1, 4096)
        return {"kind": kind, "b": _log(rng, 1, 16), "len": length, "ragged": rng.random() < 0.6,
                "new": rng.choice([1, 1, length]), "heads": heads, "dim": dim, "page": page,
                "dt": rng.choice(["bf16", "bf16", "f32"]), "method": rng.choice(["sweep", "absmax"])}
    group = rng.choice([1, 2, 4, 4, 7, 8])
    new = rng.choice([1, 1, 1, 2, 4, _log(rng, 5, 1024)])
    most = max(1, 16384 // (group * new)) if new < 5 else max(1, 2048 // new)
    b = _log(rng, 1, min(64, most))
    if kind == "attend":
        return {"kind": kind, "b": b, "len": max(new, _log(rng, 1, max(2, min(65536, 262144 // b) if new < 5 else 8192 // b))),
                "ragged": rng.random() < 0.6, "new": new, "heads": heads, "group": group, "dim": dim, "page": page}
    return {"kind": kind, "prefix": _log(rng, 100, 32768 if new < 5 else 4096), "b": b, "len": max(new, _log(rng, 1, 1000)),
            "ragged": rng.random() < 0.7, "new": new, "heads": heads, "group": group, "dim": dim, "page": page}


# --------------------------------------------------------------------------- sizes
def _lens(case):
    """Cached tokens of each sequence (its own pages), and how many of them are new."""
    b, n = case["b"], case["len"]
    lens = [n - (i * 7919 + (i * i * 104729) % 5) % n if case["ragged"] else n for i in range(b)]
    return lens, [min(v, case["new"] - (i % 2 if case["ragged"] and case["new"] > 1 else 0)) for i, v in enumerate(lens)]


def _offsets(counts):
    at = [0]
    for n in counts:
        at.append(at[-1] + n)
    return at


def _freqs(case):
    """Radians a position for each pair; with a factor, slow ones (under 1 turn in 8192 positions) are divided by it, fast
    ones (over 4) stay, those between in proportion."""
    f = [10000.0 ** (-2.0 * i / case["rot"]) for i in range(case["rot"] // 2)]
    if case["factor"] == 1.0:
        return f
    ramp = [min(1.0, max(0.0, (8192 * v / (2 * math.pi) - 1.0) / 3.0)) for v in f]
    return [v * ((1 - r) / case["factor"] + r) for v, r in zip(f, ramp)]


def _magnitude(case):
    return 0.1 * math.log(case["factor"]) + 1.0


# --------------------------------------------------------------------------- inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, *shape):
    return torch.randn(*shape, device="cuda", generator=g)


def _ints(v, dtype=torch.int32):
    return torch.tensor(v, dtype=dtype, device="cuda")


def _table(lens, page, first, total, g):
    """Pages of each sequence in an order of the pool's own; entries behind a sequence's last page are -1."""
    counts = [-(-n // page) for n in lens]
    ids = first + torch.randperm(total - first, device="cuda", generator=g)[:sum(counts)].int()
    used = torch.arange(max(counts + [1]), device="cuda")[None, :] < _ints(counts)[:, None]
    table = torch.full(used.shape, -1, dtype=torch.int32, device="cuda")
    table[used] = ids
    return table


def _slots(table, lens, new, page):
    """The place in the pool of each new token: page * size + offset, sequence after sequence."""
    where = [(b, j) for b, (n, k) in enumerate(zip(lens, new)) for j in range(n - k, n)]
    b, j = _ints([w[0] for w in where], torch.int64), _ints([w[1] for w in where], torch.int64)
    return table[b, j // page].long() * page + j % page


def _pool(pages, heads, page, dim, g):
    """A cache as earlier steps have left it: K and V by block maximum."""
    codes = torch.empty(pages, heads, 2, page, dim // 2, dtype=torch.uint8, device="cuda")
    sf = torch.empty(pages, heads, 2, dim // 16, page, dtype=torch.uint8, device="cuda")
    scale = torch.exp(0.5 * _randn(g, heads, 2, 1, 1))
    S = _randn(g, 1 << 20).abs().amax().reshape(1) * (2.0 / (6 * 256))       # as calibration finds it
    mid = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device="cuda")
    step = max(1, (1 << 26) // (heads * 2 * page * dim))
    for p in range(0, pages, step):
        n = min(step, pages - p)
        y = _randn(g, n, heads, 2, page, dim) * scale / S
        y = y.view(n, heads, 2, page, dim // 16, 16)
        sc = (y.abs().amax(-1) / 6.0).clamp(2.0 ** -9, 448.0).to(torch.float8_e4m3fn)
        t = (y / sc.float().unsqueeze(-1)).view(n, heads, 2, page, dim)
        q = torch.bucketize(t.abs(), mid).to(torch.uint8) | (torch.signbit(t).to(torch.uint8) << 3)
        codes[p:p + n] = q[..., 0::2] | (q[..., 1::2] << 4)
        sf[p:p + n] = sc.view(torch.uint8).transpose(-1, -2)
    return codes, sf, S, S.clone()


def prepare(case, seed):
    g = _gen(seed)
    s = dict(case)
    kind, dim = case["kind"], case["dim"]
    if kind == "rope":
        t, heads = case["t"], case["heads"]
        x = _randn(g, t, heads, dim) * torch.exp(0.5 * _randn(g, 1, heads, 1))
        s["x"] = x.to(TYPES[case["dt"]])
        s["y"] = torch.empty_like(s["x"])
        s["positions"] = torch.randint(0, case["far"], (t,), device="cuda", generator=g)
        freqs = _freqs(case)
        s["freqs"] = torch.tensor(freqs, dtype=torch.float64, device="cuda")
        turns = [int(math.ldexp(f / (2 * math.pi), 64)) for f in freqs]
        s["turns"] = _ints([v - (1 << 64) if v >> 63 else v for v in turns], torch.int64)
        s["magnitude"] = _magnitude(case)
        return s
    heads, page = case["heads"], case["page"]
    lens, new = _lens(case)
    common = -(-case.get("prefix", 0) // page)
    pages = common + sum(-(-n // page) for n in lens) + 3
    s["cache"] = _pool(pages, heads, page, dim, g)
    s["table"] = _table(lens, page, common, pages, g)
    s["lens"] = _ints(lens)
    at = _offsets(new)
    s["offsets"], s["tokens"], s["most"] = _ints(at), at[-1], max(new)
    if kind == "cache":
        dt = TYPES[case["dt"]]
        s["k"], s["v"] = ((_randn(g, at[-1], heads, dim) * torch.exp(0.5 * _randn(g, 1, heads, 1))).to(dt) for _ in range(2))
        s["slots"] = _slots(s["table"], lens, new, page)
        s["starts"] = _ints([n - k for n, k in zip(lens, new)])
        s["k_back"], s["v_back"] = (torch.empty(at[-1], heads, dim, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        return s
    if kind == "prefix":
        s["common"] = torch.randperm(common, device="cuda", generator=g).int()
        s["prefix_len"] = _ints([case["prefix"]])
    hq = heads * case["group"]
    s["q"] = (_randn(g, at[-1], hq, dim) * torch.exp(0.5 * _randn(g, 1, hq, 1))).to(torch.bfloat16)
    s["out"] = torch.empty_like(s["q"])
    return s


# --------------------------------------------------------------------------- the plain forms, in 32 bits
def _values(cache, table):
    """Keys and values, fp32, of the pages in table [rows, width]: two of [rows, heads, width * page, dim]."""
    codes, sf, S_k, S_v = cache
    lut = torch.tensor(E2M1 + tuple(-v for v in E2M1), device="cuda")
    at = table.clamp(min=0).long()
    c = codes[at]                                                # [rows, width, heads, 2, page, dim/2]
    q = torch.stack((lut[(c & 15).long()], lut[(c >> 4).long()]), -1).flatten(-2)
    v = sf[at].view(torch.float8_e4m3fn).float().transpose(-1, -2)
    x = q * v.repeat_interleave(16, -1)
    k, v = ((x[:, :, :, i] * S).permute(0, 2, 1, 3, 4).flatten(2, 3) for i, S in enumerate((S_k, S_v)))
    return k, v


def _rope_plain(s):
    x = s["x"].float()
    rot = s["rot"]
    ang = s["positions"].double()[:, None] * s["freqs"][None, :]
    c, n = ((f(ang) * s["magnitude"]).float()[:, None, :] for f in (torch.cos, torch.sin))
    if s["inverse"]:
        n = -n
    r = x[..., :rot]
    a, b = (r[..., 0::2], r[..., 1::2]) if s["pairs"] == "neighbours" else (r[..., :rot // 2], r[..., rot // 2:])
    a, b = a * c - b * n, a * n + b * c
    r = torch.stack((a, b), -1).flatten(-2) if s["pairs"] == "neighbours" else torch.cat((a, b), -1)
    return {"y": torch.cat((r, x[..., rot:]), -1).to(s["x"].dtype)}


def _round_e2m1(t):
    a = t.abs()
    r = torch.where(a < 2, torch.round(2 * a) / 2, torch.where(a < 4, torch.round(a), 2 * torch.round(a / 2)))
    return torch.copysign(r.clamp(max=6), t)


def _block_scales(y, method):
    """E4M3 scale codes of y [..., 16]: the block maximum over 6, or of the eleven codes around it the one of least
    squared error."""
    top = y.abs().amax(-1) / 6.0
    if method == "absmax":
        return top.clamp(2.0 ** -9, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)
    near = top.clamp(max=448.0).to(torch.float8_e4m3fn)
    floor = near.view(torch.uint8).int() - (near.float() > top).int()
    cand = (floor.unsqueeze(-1) + torch.arange(-3, 8, device=y.device)).clamp(1, 126)
    v = cand.to(torch.uint8).view(torch.float8_e4m3fn).float().unsqueeze(-1)
    q = _round_e2m1(y.unsqueeze(-2) * (1.0 / v))
    loss = (y.unsqueeze(-2).double() - (q * v).double()).square().sum(-1)
    return cand.gather(-1, loss.argmin(-1, keepdim=True)).squeeze(-1).to(torch.uint8)


def _write_plain(x, S, part, s):
    codes, sf = s["cache"][:2]
    y = (x.float() * (1.0 / S)).view(*x.shape[:2], -1, 16)
    sc = _block_scales(y, s["method"])
    t = y * (1.0 / sc.view(torch.float8_e4m3fn).float()).unsqueeze(-1)
    mid = torch.tensor([0.25, 1.25, 2.5, 5.0], device="cuda"), torch.tensor([0.75, 1.75, 3.5], device="cuda")
    # ties go to the even code: up at the borders above odd codes only
    q = torch.bucketize(t.abs(), mid[0]) + torch.bucketize(t.abs(), mid[1], right=True)
    q = (q.to(torch.uint8) | (torch.signbit(t).to(torch.uint8) << 3)).flatten(-2)
    page = codes.shape[3]
    at, off = s["slots"] // page, s["slots"] % page
    codes[at, :, part, off] = q[..., 0::2] | (q[..., 1::2] << 4)
    sf[at, :, part, :, off] = sc


def _plain(s):
    kind = s["kind"]
    if kind == "rope":
        return _rope_plain(s)
    if kind == "cache":
        _write_plain(s["k"], s["cache"][2], 0, s)
        _write_plain(s["v"], s["cache"][3], 1, s)
        k, v = _values(s["cache"], s["table"])
        j = torch.arange(k.shape[2], device="cuda")[None, :]
        new = (j >= s["starts"][:, None]) & (j < s["lens"][:, None])
        return {"k": k.transpose(1, 2)[new].to(torch.bfloat16), "v": v.transpose(1, 2)[new].to(torch.bfloat16)}
    # queries padded to [b, heads, group, most, dim]; query i of n sees keys up to len - n + i
    lens, at, most = s["lens"], s["offsets"], s["most"]
    n = at[1:] - at[:-1]
    i = torch.arange(most, device="cuda")[None, :]
    real = i < n[:, None]
    heads, group, dim = s["heads"], s["group"], s["dim"]
    q = torch.zeros(s["b"], most, heads, group, dim, device="cuda")
    q[real] = s["q"].float().view(-1, heads, group, dim)
    q = q.permute(0, 2, 3, 1, 4) * (1.0 / math.sqrt(dim))
    k, v = _values(s["cache"], s["table"])
    j = torch.arange(k.shape[2], device="cuda")
    seen = j <= (lens - n)[:, None, None] + i[:, :, None]        # [b, most, keys]
    logits = (q.flatten(2, 3) @ k.transpose(-1, -2)).unflatten(2, (group, most))
    logits = logits.masked_fill(~seen[:, None, None], -math.inf)
    if kind == "prefix":
        pk, pv = (x[0, :, :s["prefix"]] for x in _values(s["cache"], s["common"][None]))
        rows = q.permute(1, 0, 2, 3, 4).flatten(1, 3)            # [heads, b * group * most, dim]
        shared = (rows @ pk.transpose(-1, -2)).view(heads, s["b"], group, most, -1).permute(1, 0, 2, 3, 4)
        logits = torch.cat((shared, logits), -1)
    p = torch.exp(logits - logits.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True)
    if kind == "prefix":
        width = s["prefix"]
        o = p[..., width:].flatten(2, 3) @ v
        shared = p[..., :width].permute(1, 0, 2, 3, 4).flatten(1, 3) @ pv
        o = o.unflatten(2, (group, most)) + shared.view(heads, s["b"], group, most, dim).permute(1, 0, 2, 3, 4)
    else:
        o = (p.flatten(2, 3) @ v).unflatten(2, (group, most))
    return {"out": o.permute(0, 3, 1, 2, 4).flatten(2, 3)[real].to(torch.bfloat16)}


# --------------------------------------------------------------------------- the framework's calls
def _own(s):
    from paper_2606_07618_gb300 import binding as B

    kind = s["kind"]
    if kind == "rope":
        B.nvfp4_rope(s["x"], s["positions"], s["turns"], s["y"], magnitude=s["magnitude"],
                     layout=B.NVFP4_ROPE_NEIGHBOURS if s["pairs"] == "neighbours" else B.NVFP4_ROPE_HALVES,
                     inverse=s["inverse"])
        return {"y": s["y"]}
    if kind == "cache":
        B.nvfp4_kv_write(s["cache"], s["k"], s["v"], s["slots"],
                         B.NVFP4_KV_SWEEP if s["method"] == "sweep" else B.NVFP4_KV_ABSMAX)
        B.nvfp4_kv_read(s["cache"], s["table"], s["starts"], s["offsets"], s["k_back"], s["v_back"])
        return {"k": s["k_back"], "v": s["v_back"]}
    scale = 1.0 / math.sqrt(s["dim"])
    wide = s["table"].shape[1]
    if kind == "attend":
        ws = torch.empty(B.nvfp4_kv_attention_workspace(s["cache"], s["q"], s["b"], wide, s["most"]), dtype=torch.uint8,
                         device="cuda")
        B.nvfp4_kv_attention(s["q"], s["cache"], s["table"], s["lens"], s["offsets"], s["most"], scale, s["out"],
                             workspace=ws)
        return {"out": s["out"]}
    ws = torch.empty(B.nvfp4_kv_attention_workspace(s["cache"], s["q"], s["b"], wide, s["most"], s["common"].numel()),
                     dtype=torch.uint8, device="cuda")
    B.nvfp4_kv_attention_prefix(s["q"], s["cache"], s["common"], s["prefix_len"], s["table"], s["lens"], s["offsets"],
                                s["most"], scale, s["out"], workspace=ws)
    return {"out": s["out"]}


def run(state):
    return _own(state) if own else _plain(state)


# --------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    kind, dim = case["kind"], case["dim"]
    if kind == "rope":
        n = case["t"] * case["heads"]
        return {"bytes": n * dim * 2 * (2 if case["dt"] == "bf16" else 4) + 8 * case["t"], "flops": 3 * n * case["rot"]}
    heads, held = case["heads"], 0.5 + 1.0 / 16                  # bytes of a held element
    lens, new = _lens(case)
    if kind == "cache":
        n = 2 * sum(new) * heads * dim
        return {"bytes": n * ((2 if case["dt"] == "bf16" else 4) + 2 * held + 2), "flops": 0}
    prefix, rows = case.get("prefix", 0), heads * case["group"]
    pairs = sum(k * prefix + k * n - k * (k - 1) // 2 for n, k in zip(lens, new)) * rows
    return {"bytes": 2 * held * heads * dim * (prefix + sum(lens)) + 4 * sum(new) * rows * dim, "flops": 4 * pairs * dim}


# --------------------------------------------------------------------------- the definitions, in 64 bits
def _two64(e):
    """2^e from its bits."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _e4m3_64(code):
    s = code.to(torch.int64)
    e, f = s >> 3, (s & 7).double()
    return torch.where(e == 0, f * 2.0 ** -9, (1 + f / 8) * _two64(e - 7))


def _page64(s, ids, part, S):
    """K (part 0) or V of the pages ids, one after the other, [heads, tokens, dim]: each code's sign, exponent, mantissa."""
    codes, sf = s["cache"][0][ids.long(), :, part], s["cache"][1][ids.long(), :, part]
    n, heads, page, half = codes.shape
    x = torch.empty(n, heads, page, 2 * half, dtype=torch.float64, device=codes.device)
    for k, c in enumerate((codes & 15, codes >> 4)):
        c = c.to(torch.int64)
        e, f = (c >> 1) & 3, (c & 1).double()
        mag = torch.where(e == 0, 0.5 * f, (1 + 0.5 * f) * _two64(e - 1))
        x[..., k::2] = torch.where(c >= 8, -mag, mag)
    v = _e4m3_64(sf).permute(0, 1, 3, 2) * S.double()
    for k in range(2 * half // 16):
        x[..., 16 * k:16 * k + 16] *= v[..., k:k + 1]
    return x.permute(1, 0, 2, 3).reshape(heads, n * page, 2 * half)


def _nearest64(y):
    """Of the eight magnitudes the nearest one to |y|, of two the even code."""
    a = y.abs()
    best, far = torch.zeros_like(a), a.clone()
    for code, v in enumerate(E2M1[1:], 1):
        dist = (a - v).abs()
        take = (dist < far) | ((dist == far) & (code % 2 == 0))
        best, far = torch.where(take, torch.full_like(a, v), best), torch.where(take, dist, far)
    return torch.where(torch.signbit(y), -best, best)


def _held64(x, S, method):
    """What x stands for once it is held.  Three roundings to 32 bits are part of the format's definition (they decide the
    ties, which values of few bits meet often): E = 1/S, y = x E and t = y (1/v); the rest is in 64 bits."""
    E = (1.0 / S.double()).float().double()
    y = (x.double() * E).float().double().reshape(-1, 16)
    top = (y.abs().amax(-1) / 6.0).float().double()
    grid = _e4m3_64(torch.arange(127, device=x.device))
    inverse = torch.cat((grid[:1], (1.0 / grid[1:]).float().double()))

    def elements(code):
        t = (y * inverse[code].unsqueeze(-1)).float().double()
        return _nearest64(t) * grid[code].unsqueeze(-1)

    if method == "absmax":
        top = top.clamp(max=448.0)
        up = torch.searchsorted(grid, top).clamp(1, 126)
        dl, du = top - grid[up - 1], grid[up] - top
        code = torch.where((dl < du) | ((dl == du) & (up % 2 == 1)), up - 1, up).clamp(min=1)
    else:
        first = torch.searchsorted(grid, top, right=True) - 1
        least, code = torch.full_like(top, math.inf), torch.ones_like(first)
        for d in range(-3, 8):
            c = (first + d).clamp(1, 126)
            loss = (y - elements(c)).square().sum(-1)
            code, least = torch.where(loss < least, c, code), torch.minimum(loss, least)
    return (elements(code) * S.double()).view(x.shape)


def exact(case, seed):
    kind = case["kind"]
    if kind not in ("rope", "cache") and work(case)["flops"] > 1e12:
        return None
    s = prepare(case, seed)
    if kind == "rope":
        rot, half = case["rot"], case["rot"] // 2
        y = s["x"].double()
        x = y.clone()
        for p in range(half):
            i, j = (2 * p, 2 * p + 1) if case["pairs"] == "neighbours" else (p, p + half)
            t = s["positions"].double() * _freqs(case)[p] * (-1.0 if case["inverse"] else 1.0)
            c, n = _magnitude(case) * torch.cos(t)[:, None], _magnitude(case) * torch.sin(t)[:, None]
            y[..., i] = c * x[..., i] - n * x[..., j]
            y[..., j] = n * x[..., i] + c * x[..., j]
        return {"y": y}
    if kind == "cache":
        return {"k": _held64(s["k"], s["cache"][2], case["method"]), "v": _held64(s["v"], s["cache"][3], case["method"])}
    heads, group, dim, page = case["heads"], case["group"], case["dim"], case["page"]
    lens, new = _lens(case)
    at = _offsets(new)
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    prefix = case.get("prefix", 0)
    if prefix:
        pk, pv = (_page64(s, s["common"], part, s["cache"][2 + part])[:, :prefix] for part in (0, 1))
    for b in range(case["b"]):
        ids = s["table"][b, :-(-lens[b] // page)]
        k, v = (_page64(s, ids, part, s["cache"][2 + part])[:, :lens[b]] for part in (0, 1))
        if prefix:
            k, v = torch.cat((pk, k), 1), torch.cat((pv, v), 1)
        q = s["q"][at[b]:at[b + 1]].double().view(new[b], heads, group, dim)
        last = prefix + lens[b] - new[b] + torch.arange(new[b], device="cuda")
        hide = torch.arange(k.shape[1], device="cuda")[None, :] > last[:, None]
        for h in range(heads):
            z = torch.einsum("ngd,kd->gnk", q[:, h], k[h]) / math.sqrt(dim)
            p = torch.softmax(z.masked_fill(hide, -math.inf), -1)
            out[at[b]:at[b + 1], h * group:(h + 1) * group] = torch.einsum("gnk,kd->ngd", p, v[h])
    return {"out": out}
