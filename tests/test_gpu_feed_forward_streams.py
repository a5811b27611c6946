"""One block of feed_forward.py from two streams at a time: the results of calls one after the other."""
import pytest
import torch

import fp4_reference as R

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def F():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2606_07618_gb300 import feed_forward
    return feed_forward


def block(F, fmt, f, d):
    g = torch.Generator().manual_seed(1)
    return F.GatedFeedForward(*((s[1] ** -0.5 * torch.randn(*s, generator=g)).to(torch.bfloat16).to(DEV)
                                for s in ((f, d), (f, d), (d, f))), fmt=fmt)


def inputs(t, d, n):
    """Tokens whose largest magnitudes, and with them NVFP4's global scales, are octaves apart."""
    g = torch.Generator().manual_seed(2)
    return [(4.0 ** i * torch.randn(t, d, generator=g)).to(torch.bfloat16).to(DEV) for i in range(n)]


@pytest.mark.parametrize("fmt", [R.NV, R.MX])
def test_two_streams_through_one_block(F, fmt):
    t, f, d = 300, 416, 256                                      # past the sizes that need no workspace
    ff, xs = block(F, fmt, f, d), inputs(t, d, 4)
    want = [ff(x) for x in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for i in range(40):
        with torch.cuda.stream(streams[i % 2]):
            got.append(ff(xs[i % 4]))
    torch.cuda.synchronize()
    assert all(torch.equal(y, want[i % 4]) for i, y in enumerate(got)) and ff.status.item() == 0


@pytest.mark.parametrize("fmt", [R.NV, R.MX])
def test_gradients_of_calls_made_on_two_streams(F, fmt):
    """Each stream's gradients are of its own call, though both were made before either gradient."""
    t, f, d = 130, 160, 128
    ff, xs = block(F, fmt, f, d), inputs(t, d, 2)
    dy = torch.randn(t, d, generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).to(DEV)
    want = []
    for x in xs:
        ff(x)
        want.append(ff.backward(dy))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(10):
        saved, got = [], []
        for s, x in zip(streams, xs):
            with torch.cuda.stream(s):
                ff(x)
                saved.append(ff.saved)
        for s, of in zip(streams, saved):
            with torch.cuda.stream(s):
                got.append(ff.backward(dy, saved=of))
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            assert all(torch.equal(g[k], w[k]) for k in w)
