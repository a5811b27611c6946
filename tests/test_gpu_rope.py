"""Rotary positions and their gradient against 64 bits."""
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


def freqs(turns):
    return turns.cpu().double() * (2 * math.pi / 2.0 ** 64)


def tolerance(x, dt, magnitude):
    """Two products and their sum in fp32 of factors that are off by half a step and the angle's error (2^-25 of half a turn, the
    function's own of 2 steps): 8 steps of fp32 of the pair's size; one rounding to the type."""
    size = abs(magnitude) * x.double().abs().max()
    return 8 * 2.0 ** -24 * size + (2.0 ** -8 if dt == torch.bfloat16 else 2.0 ** -24) * size * math.sqrt(2)


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("dt,tokens,heads,dim,rot", [
    (torch.bfloat16, 1, 1, 2, 2), (torch.bfloat16, 5, 3, 64, 64), (torch.float32, 7, 41, 128, 96), (torch.bfloat16, 33, 2, 128, 32),
    (torch.float32, 3, 1, 20, 6), (torch.bfloat16, 2, 2, 70, 70), (torch.bfloat16, 2000, 40, 128, 128), (torch.float32, 9, 5, 1024, 1024),
    (torch.bfloat16, 4, 2, 64, 0)])
def test_against_64_bits(B, layout, inverse, dt, tokens, heads, dim, rot):
    g = torch.Generator().manual_seed(tokens)
    x = torch.randn(tokens, heads, dim, generator=g).to(dt).cuda()
    pos = torch.randint(-2 ** 20, 2 ** 20, (tokens,), generator=g).cuda()
    turns = B.nvfp4_rope_turns(rot, 10000.0) if rot else torch.empty(0, dtype=torch.int64, device="cuda")
    out = torch.empty_like(x)
    B.nvfp4_rope(x, pos, turns, out, 1.25, layout, inverse)
    want = R.rope(x.cpu(), pos.cpu(), freqs(turns), 1.25, layout == B.NVFP4_ROPE_HALVES, inverse)
    # 2^20 positions of a frequency held in 53 bits by the reference: 2^-33 of a radian
    assert ((out.cpu().double() - want).abs() <= tolerance(x.cpu(), dt, 1.25)).all()
    assert torch.equal(out[..., rot:], x[..., rot:])
    B.nvfp4_rope(x, pos, turns, None, 1.25, layout, inverse)     # in place
    assert torch.equal(x, out)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("layout", [0, 1])
def test_strides(B, dt, layout):
    """Heads of a projection's buffer, odd strides and bases, heads first; nothing beside them is touched."""
    tokens, heads, dim = 11, 3, 64
    turns = B.nvfp4_rope_turns(dim)
    pos = torch.arange(tokens, device="cuda") * 1000
    for first, width in ((0, 400), (8, 400), (1, 401), (3, 199)):
        buf = torch.randn(tokens, width, generator=torch.Generator().manual_seed(1)).to(dt).cuda()
        x = buf[:, first:first + heads * dim].unflatten(1, (heads, dim))
        want = torch.empty(tokens, heads, dim, dtype=dt, device="cuda")
        B.nvfp4_rope(x.contiguous(), pos, turns, want, layout=layout)
        keep = buf.clone()
        B.nvfp4_rope(x, pos, turns, layout=layout)
        assert torch.equal(x, want)
        keep[:, first:first + heads * dim] = buf[:, first:first + heads * dim]
        assert torch.equal(buf, keep)
    x = torch.randn(heads, tokens, dim, device="cuda").to(dt).transpose(0, 1)
    out = torch.empty(heads, tokens, dim, device="cuda", dtype=dt).transpose(0, 1)
    B.nvfp4_rope(x, pos, turns, out, layout=layout)
    want = torch.empty(tokens, heads, dim, dtype=dt, device="cuda")
    B.nvfp4_rope(x.contiguous(), pos, turns, want, layout=layout)
    assert torch.equal(out, want)


def test_far_positions(B):
    """Positions past 2^40: the angle modulo a turn is exact, so two positions that differ by whole turns of a frequency agree."""
    turns = torch.tensor([2 ** 62, 2 ** 44, 1], device="cuda")  # a quarter of a turn, 2^-20 and 2^-64 of one
    x = torch.randn(3, 1, 6, device="cuda")
    pos = torch.tensor([2 ** 41 + 1, 1, -(2 ** 41) + 1], device="cuda")
    out = torch.empty_like(x)
    B.nvfp4_rope(x, pos, turns, out, layout=B.NVFP4_ROPE_NEIGHBOURS)
    same = torch.empty_like(x)
    B.nvfp4_rope(x, torch.ones(3, dtype=torch.int64, device="cuda"), turns, same, layout=B.NVFP4_ROPE_NEIGHBOURS)
    assert torch.equal(out[..., :4], same[..., :4])


@pytest.mark.parametrize("layout", [0, 1])
def test_gradient(B, layout):
    """The inverse is the transpose: against the gradient of the formula by autograd, and against differences of the call."""
    tokens, heads, dim, m = 5, 2, 16, 1.3
    g = torch.Generator().manual_seed(3)
    x, dy = (torch.randn(tokens, heads, dim, generator=g).cuda() for _ in range(2))
    turns, pos = B.nvfp4_rope_turns(dim, 500.0), torch.tensor([0, 1, 5, 77, 1000], device="cuda")
    dx = torch.empty_like(x)
    B.nvfp4_rope(dy, pos, turns, dx, m, layout, inverse=True)
    leaf = x.cpu().double().requires_grad_()
    i = torch.arange(dim // 2)
    a, b = (i, i + dim // 2) if layout else (2 * i, 2 * i + 1)
    t = (pos.cpu().double()[:, None] * freqs(turns)[None])[:, None]
    y = torch.zeros(tokens, heads, dim, dtype=torch.float64)
    y = y.index_add(2, a, m * (leaf[..., a] * t.cos() - leaf[..., b] * t.sin()))
    y = y.index_add(2, b, m * (leaf[..., a] * t.sin() + leaf[..., b] * t.cos()))
    (y * dy.cpu().double()).sum().backward()
    assert ((dx.cpu().double() - leaf.grad).abs() <= tolerance(dy.cpu(), torch.float32, m)).all()
    # the operator is linear: a difference of step h is exact but for fp32's roundings of its two sides, each half a step of
    # results below 16, and those of tolerance() twice
    f = lambda v: B.nvfp4_rope(v, pos, turns, torch.empty_like(v), m, layout).double()  # noqa: E731
    for e in (0, 3, dim - 1):
        step = torch.zeros_like(x)
        step[..., e] = 1.0
        d = ((f(x + step) - f(x - step)) / 2 * dy.double()).sum(-1)
        size = 2 * float((x.abs().max() + 1) * m)
        tol = dim * float(dy.abs().max()) * (8 + 2) * 2.0 ** -24 * size
        assert ((d - dx[..., e].double()).abs() <= tol).all()


def test_graph_and_stream(B):
    x = torch.randn(8, 4, 64, device="cuda")
    pos, turns = torch.arange(8, device="cuda"), B.nvfp4_rope_turns(64)
    out, want = torch.empty_like(x), torch.empty_like(x)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.nvfp4_rope(x, pos, turns, out)
    pos += 100
    graph.replay()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    B.nvfp4_rope(x, pos, turns, want, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out, want)
