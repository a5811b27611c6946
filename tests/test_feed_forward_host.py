"""feed_forward.py without a GPU: what it hands to the library's calls, which are replaced by ones that record."""
import ctypes

import pytest
import torch

from paper_2606_07618_gb300 import binding as B
from paper_2606_07618_gb300 import feed_forward as F

CALLS = ("mxfp4_quantize", "scalesweep_quantize_dynamic", "scalesweep_quantize_group", "fp4_gated_ff", "fp4_matmul",
         "fp4_matmul_backward", "fp4_gated_ff_backward")


@pytest.fixture
def calls(monkeypatch):
    """(name, arguments) of each call; the arguments stay alive, so that their addresses stay apart."""
    seen = []
    for name in CALLS:
        monkeypatch.setattr(B, name, lambda *a, _name=name, **k: seen.append((_name, a)))
    return seen


def block(fmt, f=64, d=32, dtype=torch.bfloat16, **kw):
    return F.GatedFeedForward(*(torch.randn(*s).to(dtype) for s in ((f, d), (f, d), (d, f))), fmt=fmt, **kw)


def test_calls_of_one_block_share_no_workspace(calls):
    """Two calls may run at one time on two streams: each has a workspace of its own for the global scale."""
    ff = block(B.FP4_FMT_NVFP4)
    for _ in range(2):
        ff(torch.randn(4, 32).to(torch.bfloat16))
    ws = [a[10] for n, a in calls if n == "scalesweep_quantize_dynamic"]
    assert len(ws) == 4 and len({w.data_ptr() for w in ws}) == 4
    assert all(w.numel() == B.nvfp4_dynamic_workspace() for w in ws)


@pytest.mark.parametrize("fmt", [B.FP4_FMT_NVFP4, B.FP4_FMT_MXFP4])
def test_backward_of_an_earlier_call(calls, fmt):
    """The operands of the call that is asked for, not those of the one made since."""
    ff = block(fmt)
    saved = []
    for t in (4, 4):
        ff(torch.randn(t, 32).to(torch.bfloat16))
        saved.append(ff.saved)
    dy = torch.zeros(4, 32, dtype=torch.bfloat16)
    for of in saved:
        del calls[:]
        ff.backward(dy, saved=of)
        got = {n: a for n, a in calls}
        assert got["fp4_matmul_backward"][1] is of[1] and got["fp4_gated_ff_backward"][2] is of[0]
    del calls[:]
    ff.backward(dy)                                              # the last call's
    assert dict(calls)["fp4_matmul_backward"][1] is saved[1][1]


@pytest.mark.parametrize("fmt", [B.FP4_FMT_NVFP4, B.FP4_FMT_MXFP4])
def test_weights_and_tokens_of_any_strides(calls, monkeypatch, fmt):
    """Transposed weights, and columns of a wider tensor, reach the quantisers as rows of consecutive elements."""
    read = []

    def group(desc, *a, **k):                                    # the copies are gone after the call
        for t in desc:
            at = (ctypes.c_uint8 * (2 * t.rows * t.cols)).from_address(t.x)
            read.append(torch.frombuffer(at, dtype=torch.bfloat16).view(t.rows, t.cols).clone())
    monkeypatch.setattr(B, "scalesweep_quantize_group", group)
    wide, x = torch.randn(64, 80).to(torch.bfloat16), torch.randn(32, 6).to(torch.bfloat16).t()
    ws = wide[:, 8:40], wide[:, 40:72], torch.randn(64, 32).to(torch.bfloat16).t()
    F.GatedFeedForward(*ws, fmt=fmt)(x)
    if fmt == B.FP4_FMT_MXFP4:
        read = [a[0] for n, a in calls if n == "mxfp4_quantize"]
        assert all(s.stride(1) == 1 for s in read)
    assert all(torch.equal(a, b) for a, b in zip(read, ws)) and len(read) >= 3


@pytest.mark.parametrize("fmt", [B.FP4_FMT_NVFP4, B.FP4_FMT_MXFP4])
def test_one_status_word(calls, fmt):
    """Every call of a block, the quantisation of its weights among them, reports in the same word."""
    at = {"mxfp4_quantize": 4, "scalesweep_quantize_dynamic": 9, "scalesweep_quantize_group": 5, "fp4_matmul": 4,
          "fp4_matmul_backward": 7, "fp4_gated_ff_backward": 11}
    ff = block(fmt)
    ff(torch.randn(4, 32).to(torch.bfloat16))
    ff.backward(torch.zeros(4, 32, dtype=torch.bfloat16))
    words = [a[at[n]] for n, a in calls if n in at]
    assert len(words) >= 6 and all(w is ff.status for w in words)
