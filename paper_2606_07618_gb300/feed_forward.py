"""A gated feed-forward block on 4-bit operands, run and tuned through the C ABI.

``GatedFeedForward`` quantises the three weights of a block once and then runs

    y = (act(x Wg^T) * (x Wu^T)) Wd^T

with every operand in 4 bits: the activations are quantised per call, the gated part and
the down product take the codes and scales as they are, and ``backward`` gives the
gradients with respect to the values the codes stand for (straight through the
quantisers).

  * MXFP4: ``mxfp4_quantize``, then ``fp4_gated_ff`` writing its result in MXFP4 already,
    then ``fp4_matmul``: three launches.
  * NVFP4: weights by ScaleSweep (one grouped call), activations by
    ``scalesweep_quantize_dynamic`` (global scale and sweep in one call), the gated result
    in bf16 and quantised the same way.

``status`` is the calls' status word on the device, which nothing here reads: the kernels set bit 0
where a weight, x or h held a NaN or an infinity (MXFP4: zeros for its block; NVFP4: a global scale
that leaves NaNs out and is infinite for an infinity) and bits 1 and 16 where a wait ran out.  A
program reads and clears it where it can wait for the GPU.

The gradients are a program's own to apply: a block does not keep the weights it was made of, takes
part in no autograd graph, and a step of tuning makes a new block of the new weights.

All work runs in the library's kernels on the current stream; this module only arranges
buffers.  A thread may call a block from several streams, each ordered after the block's
construction; what a call keeps for its gradients is ``saved`` (the last call's), which a program
that makes more calls before the ``backward`` of one takes and passes to it.
"""
from __future__ import annotations

import torch

from . import binding as B
from .step import QuantizeStep


class GatedFeedForward:
    def __init__(self, w_gate, w_up, w_down, fmt: int = B.FP4_FMT_MXFP4, act: int = B.FP4_ACT_SILU,
                 importance=None):
        """w_gate, w_up [f, d] and w_down [d, f]: bf16 or fp32 weights on the GPU, of any strides (f and d multiples of 32; not kept).
        importance: optional per-input-channel WMSE weights of the three (fp32, NVFP4 only)."""
        if fmt not in (B.FP4_FMT_NVFP4, B.FP4_FMT_MXFP4):
            raise ValueError(f"unknown format {fmt}")
        f, d = w_gate.shape
        if w_up.shape != (f, d) or w_down.shape != (d, f):
            raise ValueError(f"weights of {tuple(w_gate.shape)}, {tuple(w_up.shape)} and {tuple(w_down.shape)}")
        if f % 32 or d % 32:
            raise ValueError("both widths have to be multiples of 32")
        if importance is not None and fmt == B.FP4_FMT_MXFP4:
            raise ValueError("importance weights are NVFP4's: MXFP4 scales follow from the block maximum")
        self.fmt, self.act, self.f, self.d = fmt, act, f, d
        self.device = w_gate.device
        self.status = torch.zeros(1, dtype=torch.int32, device=self.device)
        ws = [w_gate, w_up, w_down]
        if fmt == B.FP4_FMT_MXFP4:
            self.gate, self.up, self.down = (self._quantise(w) for w in ws)
        else:
            q = QuantizeStep([w.contiguous() for w in ws], importance, objective=B.NVFP4_OBJ_MSE if importance is None else B.NVFP4_OBJ_WMSE)
            q.status = self.status
            q()
            self.gate, self.up, self.down = ((o["codes"], o["sf_swizzled"], q.S[i:i + 1]) for i, o in enumerate(q.outs))
        self.saved = None

    # the quantised x and h of the last call
    @property
    def _x(self):
        return self.saved[0]

    @property
    def _h(self):
        return self.saved[1]

    def _quantise(self, x):
        """x as an operand in this block's format."""
        rows, cols = x.shape
        codes = torch.empty(rows, cols // 2, dtype=torch.uint8, device=self.device)
        if self.fmt == B.FP4_FMT_MXFP4:
            if x.stride(1) != 1:                                 # rows may lie apart, their elements not
                x = x.contiguous()
            sf = torch.empty(B.mx_swizzled_bytes(rows, cols), dtype=torch.uint8, device=self.device)
            B.mxfp4_quantize(x, codes, None, sf, self.status)
            return codes, sf, None
        sf = torch.empty(B.swizzled_bytes(rows, cols), dtype=torch.uint8, device=self.device)
        S = torch.empty(1, device=self.device)
        # a workspace for each call: the global scale is reduced in it, and calls on two streams run at one time
        ws = torch.empty(B.nvfp4_dynamic_workspace(), dtype=torch.uint8, device=self.device)
        win = (B.NVFP4_WINDOW_DEFAULT, B.NVFP4_WINDOW_DEFAULT)
        B.scalesweep_quantize_dynamic(x.contiguous(), 16, 256.0, B.NVFP4_OBJ_MSE, None, 0, *win, S, self.status, ws,
                                      codes, None, sf)
        return codes, sf, S

    def __call__(self, x):
        """y [t, d] bf16 of x [t, d] (bf16 or fp32).  The quantised x and h stay for ``backward``, as ``saved``."""
        t = x.shape[0]
        if x.dim() != 2 or x.shape[1] != self.d:
            raise ValueError(f"x of shape {tuple(x.shape)}, [t, {self.d}] is wanted")
        qx = self._quantise(x)
        if self.fmt == B.FP4_FMT_MXFP4:
            codes = torch.empty(t, self.f // 2, dtype=torch.uint8, device=self.device)
            sf = torch.empty(B.mx_swizzled_bytes(t, self.f), dtype=torch.uint8, device=self.device)
            B.fp4_gated_ff(self.fmt, self.act, qx, self.gate, self.up, None, codes, sf, self.status)
            qh = (codes, sf, None)
        else:
            h = torch.empty(t, self.f, dtype=torch.bfloat16, device=self.device)
            B.fp4_gated_ff(self.fmt, self.act, qx, self.gate, self.up, h, status=self.status)
            qh = self._quantise(h)
        y = torch.empty(t, self.d, dtype=torch.bfloat16, device=self.device)
        B.fp4_matmul(self.fmt, qh, self.down, y, self.status)
        self.saved = qx, qh
        return y

    def backward(self, dy, weights: bool = True, saved=None) -> dict:
        """Gradients (bf16) of sum(dy * y) for the call that ``saved`` is of (None: the last one): {"x", "gate", "up",
        "down"}, or {"x"} alone for frozen weights."""
        saved = saved or self.saved
        if saved is None:
            raise RuntimeError("backward before a call")
        qx, qh = saved
        if self.device.type == "cuda":
            # they may be another stream's, and dropped by its next call before this one's kernels have read them
            for v in (*qx, *qh):
                if v is not None:
                    v.record_stream(torch.cuda.current_stream(self.device))
        t = qx[0].shape[0]
        if dy.shape != (t, self.d):
            raise ValueError(f"dy of shape {tuple(dy.shape)}, {(t, self.d)} is wanted")
        new = lambda *s: torch.empty(*s, dtype=torch.bfloat16, device=self.device)  # noqa: E731
        ws = torch.empty(max(B.fp4_matmul_backward_workspace(t, self.d, self.f),
                             B.fp4_gated_ff_backward_workspace(t, self.f, self.d)), dtype=torch.uint8, device=self.device)
        g = {"x": new(t, self.d)}
        dh = new(t, self.f)
        if weights:
            g.update(gate=new(self.f, self.d), up=new(self.f, self.d), down=new(self.d, self.f))
        B.fp4_matmul_backward(self.fmt, qh, self.down, dy, dh, g.get("down"), ws, self.status)
        B.fp4_gated_ff_backward(self.fmt, self.act, qx, self.gate, self.up, dh, g["x"], g.get("gate"), g.get("up"),
                                None, ws, self.status)
        return g


def main(t: int = 1024, f: int = 14336, d: int = 4096) -> None:
    """Runs a block of random weights in both formats: its error against fp32 weights and activations, and its times."""
    g = torch.Generator(device="cuda").manual_seed(0)
    w = [(s[1] ** -0.5 * torch.randn(*s, device="cuda", generator=g)).to(torch.bfloat16) for s in ((f, d), (f, d), (d, f))]
    x = torch.randn(t, d, device="cuda", generator=g).to(torch.bfloat16)
    dy = torch.randn(t, d, device="cuda", generator=g).to(torch.bfloat16)
    wg, wu, wd = (v.float() for v in w)
    want = (torch.nn.functional.silu(x.float() @ wg.T) * (x.float() @ wu.T)) @ wd.T
    for name, fmt in (("NVFP4", B.FP4_FMT_NVFP4), ("MXFP4", B.FP4_FMT_MXFP4)):
        block = GatedFeedForward(*w, fmt=fmt)
        err = ((block(x).float() - want).norm() / want.norm()).item()
        times = []
        for run in (lambda: block(x), lambda: block.backward(dy)):
            for _ in range(3):
                run()
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            for _ in range(10):
                run()
            b.record()
            torch.cuda.synchronize()
            times.append(a.elapsed_time(b) * 100)
        print(f"{name}: {t} tokens, {d} -> {f} -> {d}: relative error {err:.3f}, forward {times[0]:.0f} us, "
              f"gradients {times[1]:.0f} us")


if __name__ == "__main__":
    main()
