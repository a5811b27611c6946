"""include/nvfp4kv.h: every declared entry point is exported, the frequency table, and bad arguments, which are refused on the
host before any launch (no GPU needed; the pointers are never dereferenced)."""
import ctypes
import math
import os
import re

import pytest
import torch

from conftest import ROOT

FAKE = 0x10000000
OK, INVALID, UNSUPPORTED, ALIGNMENT, RANGE = 0, 1, 2, 3, 4


@pytest.fixture(scope="module")
def B():
    from paper_2606_07618_gb300 import binding
    binding.lib()
    return binding


def test_header_and_exports(B):
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "nvfp4kv.h")).read(), flags=re.S)
    names = re.findall(r"^(?:nvfp4_status|size_t)\s+([a-z0-9_]+)\s*\(", src, re.M)
    assert sorted(names) == sorted(["nvfp4_rope_turns", "nvfp4_rope", "nvfp4_kv_write", "nvfp4_kv_read", "nvfp4_kv_attention",
                                    "nvfp4_kv_attention_workspace", "nvfp4_kv_attention_prefix",
                                    "nvfp4_kv_selftest_wait_timeout"])
    for n in names:
        assert hasattr(B.lib(), n), n


# --------------------------------------------------------------------------- frequencies
def turns_of(B, *args, **kw):
    return [v / 2.0 ** 64 for v in B.nvfp4_rope_turns(*args, device="cpu", **kw).tolist()]


@pytest.mark.parametrize("rot", [2, 6, 64, 128, 1024])
def test_turns(B, rot):
    got = turns_of(B, rot, 10000.0)
    want = [10000.0 ** (-2 * i / rot) / (2 * math.pi) for i in range(rot // 2)]
    # 53 bits of the double, a power that may be a few places off; the table's multiples of 2^-64 by half of one
    assert all(abs(g - w) <= 8 * 2.0 ** -53 * w + 2.0 ** -65 for g, w in zip(got, want))


def test_scaled_turns(B):
    rot, base, f = 64, 500000.0, 8.0
    plain = turns_of(B, rot, base)
    # both sides hold multiples of 2^-64, off by half of one each
    near = lambda a, b: all(abs(x - y) <= 2.0 ** -45 * y + 2.0 ** -64 for x, y in zip(a, b))  # noqa: E731
    assert near(turns_of(B, rot, base, scaling=B.NVFP4_ROPE_LINEAR, factor=f), [v / f for v in plain])
    stretched = turns_of(B, rot, base, scaling=B.NVFP4_ROPE_BASE, factor=f)
    assert near(stretched[:1], plain[:1]) and near(stretched[-1:], [plain[-1] / f])
    assert all(a <= b for a, b in zip(stretched, plain))
    L, slow, fast = 8192.0, 1.0, 4.0
    bands = turns_of(B, rot, base, scaling=B.NVFP4_ROPE_BANDS, factor=f, original_len=L, slow=slow, fast=fast)
    for got, v in zip(bands, plain):
        if L * v >= fast:
            assert got == v
        elif L * v <= slow:
            assert near([got], [v / f])
        else:
            assert v / f < got < v
    assert near(turns_of(B, rot, base, scaling=B.NVFP4_ROPE_LINEAR, factor=1.0), plain)


def test_turns_refusals(B):
    L = B.lib()
    out = (ctypes.c_uint64 * 512)()
    t = lambda rot=64, base=10000.0, kind=0, factor=2.0, length=4096.0, slow=1.0, fast=4.0, p=out: \
        L.nvfp4_rope_turns(rot, base, kind, factor, length, slow, fast, p)
    assert t() == OK and t(kind=3) == OK and t(factor=0.0) == OK                # factor is not read without scaling
    assert t(p=None) == INVALID and t(rot=0) == INVALID and t(rot=63) == INVALID and t(rot=1026) == INVALID
    assert t(base=1.0) == INVALID and t(base=math.nan) == INVALID and t(base=math.inf) == INVALID
    assert t(kind=4) == INVALID and t(kind=-1) == INVALID
    assert t(kind=1, factor=0.5) == INVALID and t(kind=2, factor=math.nan) == INVALID and t(kind=1, factor=math.inf) == INVALID
    assert t(kind=2, rot=2) == INVALID and t(kind=2, rot=4, factor=1e300) == RANGE
    assert t(kind=3, length=0.0) == INVALID and t(kind=3, slow=-1.0) == INVALID and t(kind=3, slow=4.0) == INVALID
    assert t(kind=3, fast=math.inf) == INVALID and t(kind=3, length=math.nan) == INVALID


# --------------------------------------------------------------------------- refusals of the C calls
def test_rope_refusals(B):
    L = B.lib()
    r = lambda x=FAKE, xt=256, xh=64, out=FAKE + 0x1000000, ot=256, oh=64, dt=0, tokens=8, heads=4, dim=64, rot=64, \
        pos=FAKE + 0x2000000, turns=FAKE + 0x3000000, m=1.0, layout=1: \
        L.nvfp4_rope(x, xt, xh, out, ot, oh, dt, tokens, heads, dim, rot, pos, turns, m, layout, 0, None)
    assert r(tokens=0) == OK and r(heads=0) == OK and r(dim=0, rot=0) == OK
    assert r(dt=2) == INVALID and r(tokens=-1) == INVALID and r(heads=-1) == INVALID and r(layout=2) == INVALID
    assert r(dim=63) == INVALID and r(rot=7) == INVALID and r(rot=66) == INVALID and r(rot=-2) == INVALID
    assert r(m=math.nan) == INVALID and r(m=math.inf) == INVALID
    assert r(x=None) == INVALID and r(out=None) == INVALID and r(pos=None) == INVALID and r(turns=None) == INVALID
    assert r(xh=63) == INVALID and r(xt=255) == INVALID and r(xt=0) == INVALID and r(oh=-64) == INVALID
    assert r(x=FAKE + 1) == ALIGNMENT and r(dt=1, out=FAKE + 0x1000002) == ALIGNMENT and r(pos=FAKE + 0x2000004) == ALIGNMENT
    assert r(turns=FAKE + 0x3000004) == ALIGNMENT
    assert r(out=FAKE + 128) == INVALID and r(out=FAKE, ot=512) == INVALID       # neither apart nor the same tensor
    assert r(out=FAKE, xt=512, ot=512, oh=128, xh=64) == INVALID
    assert r(pos=FAKE + 0x1000000) == INVALID                      # positions under the result
    assert r(tokens=2 ** 31) == RANGE and r(heads=65536, xt=2 ** 23, ot=2 ** 23) == RANGE and r(dim=1026, rot=64) == RANGE
    assert r(tokens=2 ** 30, xt=2 ** 40, ot=2 ** 40) == RANGE


def cache(B, codes=FAKE, sf=FAKE + 0x8000000, sk=FAKE + 0xA000000, sv=FAKE + 0xA000010, pages=8, page=64, heads=2, dim=64):
    return ctypes.byref(B.KvCache(codes, sf, sk, sv, pages, page, heads, dim))


BAD_CACHES = [(dict(dim=32), UNSUPPORTED), (dict(dim=96), UNSUPPORTED), (dict(dim=256), UNSUPPORTED), (dict(page=8), UNSUPPORTED),
              (dict(page=48), UNSUPPORTED), (dict(page=2048), UNSUPPORTED), (dict(pages=-1), INVALID), (dict(heads=0), INVALID),
              (dict(heads=65536), RANGE), (dict(pages=2 ** 31), RANGE), (dict(pages=2 ** 31 - 1, page=1024, heads=65535), RANGE),
              (dict(codes=None), INVALID), (dict(sf=None), INVALID), (dict(sk=None), INVALID), (dict(sv=None), INVALID),
              (dict(codes=FAKE + 8), ALIGNMENT), (dict(sf=FAKE + 0x8000004), ALIGNMENT), (dict(sk=FAKE + 0xA000002), ALIGNMENT)]


def write(B, c=None, k=FAKE + 0x1000000, kt=128, kh=64, v=FAKE + 0x2000000, vt=128, vh=64, dt=0, tokens=8, slots=FAKE + 0x3000000,
          method=1, st=None):
    return B.lib().nvfp4_kv_write(c or cache(B), k, kt, kh, v, vt, vh, dt, tokens, slots, method, st, None)


def read(B, c=None, table=FAKE + 0x5000000, ld=8, width=8, starts=None, offsets=FAKE + 0x6000000, batch=2, k=FAKE + 0x1000000, kt=128,
         kh=64, v=FAKE + 0x2000000, vt=128, vh=64, dt=0, tokens=8, st=None):
    return B.lib().nvfp4_kv_read(c or cache(B), table, ld, width, starts, offsets, batch, k, kt, kh, v, vt, vh, dt, tokens, st, None)


def attend(B, c=None, q=FAKE + 0x1000000, qt=256, qh=64, tokens=8, heads=4, table=FAKE + 0x5000000, ld=8, width=8,
           lens=FAKE + 0x6000000, offsets=FAKE + 0x6100000, batch=2, max_q=8, scale=0.1, out=FAKE + 0x2000000, ot=256, oh=64, lse=None,
           st=None, ws=FAKE + 0x20000000, ws_bytes=2 ** 40, prefix=None):
    if prefix is None:
        return B.lib().nvfp4_kv_attention(c or cache(B), q, qt, qh, tokens, heads, table, ld, width, lens, offsets, batch, max_q, scale,
                                          1, out, ot, oh, lse, st, ws, ws_bytes, None)
    pages, n, length = prefix
    return B.lib().nvfp4_kv_attention_prefix(c or cache(B), q, qt, qh, tokens, heads, pages, n, length, table, ld, width, lens, offsets,
                                             batch, max_q, scale, 1, out, ot, oh, lse, st, ws, ws_bytes, None)


@pytest.mark.parametrize("call", [write, read, attend])
@pytest.mark.parametrize("bad,status", BAD_CACHES)
def test_bad_caches(B, call, bad, status):
    assert call(B, c=cache(B, **bad)) == status


def test_write_refusals(B):
    w = lambda **kw: write(B, **kw)
    assert w(tokens=0) == OK
    assert w(dt=2) == INVALID and w(method=2) == INVALID and w(tokens=-1) == INVALID and w(tokens=2 ** 31) == RANGE
    assert w(k=None, v=None) == INVALID and w(slots=None) == INVALID
    assert w(kh=63) == INVALID and w(vt=127) == INVALID and w(vt=0) == INVALID
    assert w(k=FAKE + 0x1000001) == ALIGNMENT and w(dt=1, v=FAKE + 0x2000002) == ALIGNMENT and w(slots=FAKE + 0x3000004) == ALIGNMENT
    assert w(st=FAKE + 0x7000002) == ALIGNMENT
    assert w(k=FAKE + 0x100) == INVALID and w(v=FAKE + 0x8000100) == INVALID      # tokens in the pool
    assert w(slots=FAKE + 0x40) == INVALID and w(st=FAKE) == INVALID


def test_read_refusals(B):
    r = lambda **kw: read(B, **kw)
    assert r(tokens=0) == OK and r(batch=0) == OK
    assert r(dt=2) == INVALID and r(tokens=-1) == INVALID and r(batch=-1) == INVALID and r(width=-1) == INVALID
    assert r(ld=7) == INVALID and r(table=None) == INVALID and r(offsets=None) == INVALID and r(k=None, v=None) == INVALID
    assert r(table=FAKE + 0x5000002) == ALIGNMENT and r(offsets=FAKE + 0x6000002) == ALIGNMENT
    assert r(starts=FAKE + 0x6000102) == ALIGNMENT
    assert r(width=2 ** 31, ld=2 ** 31) == RANGE and r(batch=2 ** 31) == RANGE and r(tokens=2 ** 31) == RANGE
    assert r(v=FAKE + 0x1000010) == INVALID                        # k and v over one another
    assert r(k=FAKE) == INVALID and r(v=FAKE + 0x5000000) == INVALID and r(st=FAKE + 0x1000000) == INVALID
    # beside one another in one buffer they pass this check (and fail the next, which looks the pointers up)
    assert r(k=FAKE + 0x1000000, kt=512, v=FAKE + 0x1000000 + 256, vt=512) == INVALID


@pytest.mark.parametrize("prefix", [None, (FAKE + 0x6200000, 4, FAKE + 0x6300000)])
def test_attention_refusals(B, prefix):
    a = lambda **kw: attend(B, **{"prefix": prefix, **kw})
    assert a(tokens=0) == OK and a(batch=0) == OK and a(max_q=0) == OK
    assert a(tokens=-1) == INVALID and a(batch=-1) == INVALID and a(max_q=-1) == INVALID
    assert a(heads=0) == INVALID and a(heads=3) == INVALID and a(heads=65538, qt=2 ** 23, ot=2 ** 23) == RANGE
    assert a(scale=-0.1) == INVALID and a(scale=math.nan) == INVALID and a(scale=math.inf) == INVALID
    assert a(lens=None) == INVALID and a(offsets=None) == INVALID and a(table=None) == INVALID and a(q=None) == INVALID
    assert a(out=None) == INVALID and a(ld=7) == INVALID and a(qt=255) == INVALID and a(oh=32) == INVALID
    assert a(q=FAKE + 0x1000001) == ALIGNMENT and a(lens=FAKE + 0x6000002) == ALIGNMENT and a(lse=FAKE + 0x7000002) == ALIGNMENT
    assert a(width=2 ** 31, ld=2 ** 31) == RANGE and a(tokens=2 ** 31) == RANGE and a(batch=2 ** 31) == RANGE
    assert a(out=FAKE + 0x1000000) == INVALID                      # over q
    assert a(out=FAKE) == INVALID and a(lse=FAKE + 0x1000000) == INVALID and a(st=FAKE + 0x2000000) == INVALID
    if prefix:
        assert a(prefix=(None, 4, prefix[2])) == INVALID and a(prefix=(prefix[0], 4, None)) == INVALID
        assert a(prefix=(prefix[0], -1, prefix[2])) == INVALID and a(prefix=(prefix[0], 2 ** 31, prefix[2])) == RANGE
        assert a(prefix=(prefix[0] + 2, 4, prefix[2])) == ALIGNMENT and a(prefix=(prefix[0], 4, prefix[2] + 2)) == ALIGNMENT
        assert a(ws=None) == INVALID and a(ws_bytes=100) == INVALID and a(ws=FAKE + 0x20000080) == ALIGNMENT
        assert a(ws=FAKE) == INVALID


@pytest.mark.parametrize("page", [16, 64, 512, 1024])
def test_longest_tables(B, page):
    """width * page up to 2^31 - 2048 tokens, of a sequence's pages and of a prefix's: past that the kernels' token numbers, which look
    ahead of the last one, would not fit 31 bits.  (What is accepted goes on to the check that looks the pointers up, and fails that.)"""
    most = (2 ** 31 - 2048) // page
    c, pre = cache(B, page=page), lambda n: (FAKE + 0x100000000, n, FAKE + 0x6300000)  # noqa: E731
    far = dict(c=c, table=FAKE + 0x40000000, ws=FAKE + 0x200000000)
    assert attend(B, batch=1, width=most, ld=most, **far) == INVALID
    assert attend(B, batch=1, width=most + 1, ld=most + 1, **far) == RANGE
    assert attend(B, prefix=pre(most), **far) == INVALID and attend(B, prefix=pre(most + 1), **far) == RANGE
    size = lambda w, n: B.lib().nvfp4_kv_attention_workspace(c, 1, 4, 1, w, 1, n)  # noqa: E731
    assert size(most, 0) > 0 and size(most + 1, 0) == 0 and size(8, most) > 0 and size(8, most + 1) == 0


def test_selftest_refusals(B):
    L = B.lib()
    t = lambda heads=40, st=FAKE + 0x7000000: L.nvfp4_kv_selftest_wait_timeout(
        cache(B), FAKE + 0x1000000, 64 * heads, 64, 8, heads, FAKE + 0x5000000, 8, 8, FAKE + 0x6000000, FAKE + 0x6100000, 2, 8, 0.1, 1,
        FAKE + 0x2000000, 64 * heads, 64, None, st, FAKE + 0x20000000, 2 ** 40, None)
    assert t(st=None) == INVALID and t(heads=4) == UNSUPPORTED     # 16 rows: no such waits


# --------------------------------------------------------------------------- refusals of the binding
def _cache(pages=3, heads=2, page=16, dim=64):
    return (torch.zeros(pages, heads, 2, page, dim // 2, dtype=torch.uint8), torch.zeros(pages, heads, 2, dim // 16, page, dtype=torch.uint8),
            torch.ones(1), torch.ones(1))


def test_binding_checks_caches(B):
    k = torch.zeros(4, 2, 64)
    slots = torch.zeros(4, dtype=torch.int64)
    c = _cache()
    for bad, kind in (((c[0][..., :16], *c[1:]), ValueError), ((c[0], c[1][:2], *c[2:]), ValueError),
                      ((c[0].float(), *c[1:]), TypeError), ((c[0], c[1], c[2].double(), c[3]), TypeError),
                      ((c[0], c[1], c[2], torch.ones(2)), TypeError),
                      ((c[0].transpose(0, 1).contiguous().transpose(0, 1), *c[1:]), ValueError)):
        with pytest.raises(kind):
            B.nvfp4_kv_write(bad, k, k, slots)


@pytest.mark.parametrize("causal", [None, 0, 1, 2, True, "yes"])
def test_causal_is_a_truth_value(B, causal, monkeypatch):
    """Whatever is false or true in Python: the calls get 0 or 1."""
    seen = {}

    class Library:
        def __getattr__(self, name):
            return lambda *args: seen.setdefault(name, args) and 0
    monkeypatch.setattr(B, "_lib", Library())
    monkeypatch.setattr(B, "_stream", lambda stream: 0)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    q, table = torch.zeros(4, 6, 64, dtype=torch.bfloat16), torch.zeros(2, 3, dtype=torch.int32)
    args = (table, i32(1, 1), i32(0, 2, 4), 2, 0.125, q.clone(), causal)
    B.nvfp4_kv_attention(q, _cache(), *args)
    B.nvfp4_kv_attention_prefix(q, _cache(), i32(0), i32(1), *args)
    for name in ("nvfp4_kv_attention", "nvfp4_kv_attention_prefix"):
        at = seen[name].index(0.125) + 1
        assert type(seen[name][at]) is int and seen[name][at] == (1 if causal else 0)


def test_binding_checks_tensors(B):
    c = _cache()
    k = torch.zeros(4, 2, 64)
    slots = torch.zeros(4, dtype=torch.int64)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    table = torch.zeros(2, 3, dtype=torch.int32)
    for args, kind in (((k[:, :1], k, slots), ValueError), ((k, k[:3], slots), ValueError), ((k, k.bfloat16(), slots), ValueError),
                       ((None, None, slots), ValueError), ((k.half(), None, slots), TypeError), ((k, k, slots.int()), TypeError),
                       ((k, k, slots[:3]), ValueError), ((k[..., ::2].repeat(1, 1, 2)[..., ::2], None, slots), ValueError),
                       ((k.transpose(0, 2), None, slots), ValueError)):
        with pytest.raises(kind):
            B.nvfp4_kv_write(c, *args)
    for args, kind in (((table.long(), None, i32(0, 1, 2)), TypeError), ((table[0], None, i32(0, 1, 2)), ValueError),
                       ((table, i32(0), i32(0, 1, 2)), ValueError), ((table, None, i32(0, 1)), ValueError),
                       ((table.t(), None, i32(0, 1, 2, 3)), ValueError)):
        with pytest.raises(kind):
            B.nvfp4_kv_read(c, *args, k, k)
    q = torch.zeros(4, 6, 64, dtype=torch.bfloat16)
    lens, offsets = i32(1, 1), i32(0, 2, 4)
    good = (q, c, table, lens, offsets, 2, 0.1, q.clone())
    for at, v, kind in ((0, q.float(), TypeError), (7, q.float(), TypeError), (0, q[..., :32], ValueError), (7, q[:3], ValueError),
                        (0, q[:, :5], ValueError), (3, lens[:1], ValueError), (3, lens.long(), TypeError), (4, offsets[:2], ValueError)):
        bad = list(good)
        bad[at] = v
        if at == 0 and v.shape[1] == 5:
            bad[7] = v.clone()
        with pytest.raises(kind):
            B.nvfp4_kv_attention(*bad)
    with pytest.raises(ValueError):
        B.nvfp4_kv_attention(*good, lse=torch.zeros(4, 5))
    with pytest.raises(TypeError):
        B.nvfp4_kv_attention(*good, lse=torch.zeros(4, 6, dtype=torch.float64))
    with pytest.raises(TypeError):
        B.nvfp4_kv_attention_prefix(q, c, i32(0).long(), i32(1), *good[2:])
    x, pos, turns = torch.zeros(4, 2, 8), torch.zeros(4, dtype=torch.int64), torch.zeros(4, dtype=torch.int64)
    for args, kind in (((x, pos.int(), turns), TypeError), ((x, pos[:3], turns), ValueError), ((x, pos, turns.int()), TypeError),
                       ((x[0], pos, turns), ValueError), ((x.half(), pos, turns), TypeError), ((x, pos, turns, x.bfloat16()), TypeError),
                       ((x, pos, turns, x[:3]), ValueError)):
        with pytest.raises(kind):
            B.nvfp4_rope(*args)
