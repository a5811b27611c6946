"""Attention over the NVFP4 cache for finite logits of any size: the largest key takes all the weight, keys that tie share it."""
import math

import pytest
import torch

import kv_reference as R
import test_gpu_kv_paths as T

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2606_07618_gb300 import binding
    binding.lib()
    return binding


def one_hot(s, rows, exponent, seed=5):
    """Queries of one element +-2^e: a logit is that times a key's element, which has at most 6 significant bits, so scores are exact
    and differ by 2^-6 of themselves or not at all."""
    g = torch.Generator().manual_seed(seed)
    n, heads, dim = s.q.shape
    q = torch.zeros(n, heads, dim, dtype=torch.float64)
    at = torch.randint(0, dim, (n, heads, 1), generator=g)
    q.scatter_(2, at, (1 - 2 * torch.randint(0, 2, (n, heads, 1), generator=g)).double() * 2.0 ** exponent)
    s.q[rows] = q.to(torch.bfloat16)[rows]


def check_large(s, got, lse, want, rows):
    """A row's visible keys either tie with the largest or lie 2^-6 of it lower, hundreds and more: their weights are 1 / ties and 0.
    Values are exact; the sum of ties has up to `keys` roundings of fp32, the quotient and products a few, the result one of bf16.
    Past logits of 2^20 ties' weights are exactly 2^7.  Below it they are 2^(7 + d), d the rounding of the logit (2^-5 at most) and of
    the exponent's addend (2^-4): no power of two, so fp16 rounds each by up to 2^-11, all of them alike, and their fp32 sum not.  The
    quotient is off by that 2^-11.  lse is a product of five factors and a sum, each rounded once."""
    out, ref, mag, _, _ = want
    got, lse = got.double().cpu().view(out.shape)[rows], lse.double().cpu().view(ref.shape)[rows]
    out, ref, mag = out[rows], ref[rows], mag[rows]
    keys = max(s.lens) + s.prefix
    tol = 2.0 ** -8 * out.abs() + (2.0 ** -11 + (keys + 16) * 2.0 ** -24) * mag
    bad = ~((got - out).abs() <= tol)
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} off, {int(torch.isnan(got).sum())} of them NaN"
    empty = torch.isinf(ref)
    assert torch.equal(empty, lse == -math.inf)
    # logits of 0 (a key's element is 0 where the others' are below it) leave ln of the ties
    assert ((lse - ref).abs() <= 2.0 ** -20 * ref.abs() + 2.0 ** -18)[~empty].all()


def check_mixed(s, B, causal, large):
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out, lse = s.run(B, causal, status=status)
    want = s.want(causal)
    check_large(s, out, lse, want, large)
    rest = ~large
    if rest.any():
        R.check(out[rest.cuda()], [w[rest] for w in want], lse[rest.cuda()])
    assert status.item() == 0


@pytest.mark.parametrize("exponent", [24, 31, 34, 41, 100, 120])
@pytest.mark.parametrize("args,path", T.PATHS, ids=[f"{i}-{p[0]}-{p[1]}-{p[2]}" for i, (_, p) in enumerate(T.PATHS)])
def test_large_queries(B, args, path, exponent):
    """Every path; rows of ordinary size between them."""
    if path[0] == 512 and exponent not in (24, 34):
        pytest.skip("the larger shapes at two sizes")
    s = R.Setting(*args[0], **args[1], seed=7)
    large = torch.arange(s.total) % 3 != 1
    one_hot(s, large, exponent)
    check_mixed(s, B, True, large)


@pytest.mark.parametrize("queries", [1, 4, 30])
@pytest.mark.parametrize("dim", [64, 128])
def test_large_scale(B, queries, dim):
    """The scale of the logits, not the queries, is what is large."""
    s = R.Setting([333, 90], [queries, 1], 2, 3, dim, 16, seed=8)
    large = torch.ones(s.total, dtype=torch.bool)
    one_hot(s, large, 0)
    s.scale = 2.0 ** 38
    check_mixed(s, B, False, large)


@pytest.mark.parametrize("queries", [1, 4, 30, 200])
def test_dense_queries(B, queries):
    """Logits around the size from which weights are formed another way (2^20) and far past it: finite, and within the logits' error."""
    for e in (14, 17, 18, 19, 20, 22, 26, 33):
        s = R.Setting([700, 90], [queries, 1], 1, 4, 128, 16, seed=e, spread=0.3)
        s.q = (s.q.double() * 2.0 ** e).to(torch.bfloat16)
        out, lse = s.run(B)
        assert torch.isfinite(out).all() and torch.isfinite(lse).all()
        want = s.want()
        # a row's values bound its result whatever the weights are
        v = torch.cat([R.tokens_of(R.values(s.cache, 1), s.table[b], n).abs().amax() * torch.ones(m) for b, (n, m) in enumerate(zip(s.lens, s.queries))])
        assert (out.double().cpu().abs().amax((1, 2)) <= v * (1 + 2.0 ** -7)).all()
        R.check(out, want, lse)


def test_maximum_that_keeps_growing(B):
    """Keys that rise with their position, so that the maximum is followed again and again, at every size of logits."""
    for dim in (64, 128):
        for queries in (1, 4, 40):
            s = R.Setting([1300], [queries], 1, 3, dim, 16, seed=3)
            # element 0 of every key: 6 times scales that rise from 2^-6 by a step of E4M3 every 16 tokens
            codes, sf = s.cache[0], s.cache[1]
            for j in range(1300):
                page, at = int(s.table[0, j // 16]), j % 16
                codes[page, :, 0, at, 0] = 0x07 | int(codes[page, 0, 0, at, 0]) & 0xF0
                sf[page, :, 0, 0, at] = 0x10 + j // 16
            for e in (3, 20, 24, 34):
                s.q[:] = 0
                s.q[..., 0] = 2.0 ** e
                want = s.want()
                out, lse = s.run(B)
                if e < 20:
                    R.check(out, want, lse)
                else:
                    check_large(s, out, lse, want, torch.ones(s.total, dtype=torch.bool))


@pytest.mark.parametrize("queries", [1, 4, 30, 200])
def test_not_finite_beside_large(B, queries):
    """A NaN and infinities stay in their rows where other rows' logits are large."""
    s = R.Setting([700, 90], [queries, 1], 1, 4, 128, 16, seed=9)
    large = torch.ones(s.total, dtype=torch.bool)
    one_hot(s, large, 40)
    q = s.q.cuda()
    nan = torch.zeros(s.total, 4, dtype=torch.bool)
    for row, head, value in ((0, 1, math.nan), (0, 3, math.inf), (s.total - 1, 0, -math.inf)):
        q[row, head, 5:7] = value
        nan[row, head] = True
    out, lse = s.run(B, q=q)
    # an infinity times a key's 0 is NaN, times others infinite: the row is NaN or, where every score is -inf, 0; the others are as ever
    want = s.want()
    for t in (out, lse, *want):
        t.view(s.total, 4, -1)[nan.to(t.device)] = 0
    check_large(s, out, lse, want, large)
