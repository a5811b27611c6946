"""A key/value cache in NVFP4 for serving: pages, steps of a batch, and what each layer does in a step.

``Pages`` keeps the books of a pool of pages on the host: which sequence holds which pages and how many tokens.  It is
the same for all layers of a model.  Each forward pass takes one ``step`` of it, the device tensors that say where the
batch's new tokens go and what their queries see.  ``KVCache`` is one layer's pool: it writes a step's keys and values as
4-bit blocks, answers its queries and reads tokens back.  ``Rotary`` turns queries and keys before that.

    pages, rotary = Pages(1024, 64), Rotary(128, base=500000.0)
    caches = [KVCache(pages, heads=8, dim=128, S_k=..., S_v=...) for _ in range(layers)]
    a, b = pages.add(), pages.add()
    step = pages.step([(a, 700), (b, 1)])            # 700 new tokens of a, one of b
    for cache in caches:
        rotary(qk, step.positions)                   # query and key heads side by side, in place
        cache.write(step, k, v)
        out = cache.attend(step, q)

Sequences that begin with the same prompt share it: ``pages.share(a)`` makes what a holds a prefix, and a step of
sequences that were added with that prefix attends to it once for all of them.

All arithmetic runs in the library's kernels on the current stream; this module only arranges buffers.  ``status`` of a cache is
the calls' status word on the device, which nothing here reads: bit 0 where a written token was not finite, bits 2 and 4 where
a step did not fit the cache or a wait ran out.
"""
from __future__ import annotations

import math

import torch

from . import binding as B


class Prefix:
    """The pages and tokens of a prompt that several sequences share; pages is None once it is dropped."""

    def __init__(self, pages, length: int):
        self.pages, self.length, self.users = pages, length, 0


class _Sequence:
    def __init__(self, prefix):
        self.pages, self.length, self.prefix = [], 0, prefix


class Step:
    """One pass of a batch: table [sequences, pages], lens, offsets, slots and positions on the device, rows of q (tokens), the most
    queries of a sequence, and the prefix's pages and length or None."""

    def __init__(self, table, lens, offsets, slots, positions, tokens, max_q, prefix, prefix_len):
        self.table, self.lens, self.offsets, self.slots, self.positions = table, lens, offsets, slots, positions
        self.tokens, self.max_q, self.prefix, self.prefix_len = tokens, max_q, prefix, prefix_len


class Pages:
    def __init__(self, count: int, size: int = 64, device="cuda"):
        if size < 16 or size > 1024 or size & (size - 1):
            raise ValueError(f"pages of a power of two from 16 to 1024 tokens are wanted, not {size}")
        if count < 0:
            raise ValueError(f"{count} pages")
        self.count, self.size, self.device = count, size, torch.device(device)
        self.free = list(range(count - 1, -1, -1))
        self.sequences = {}
        self.next = 0

    def add(self, prefix: Prefix | None = None) -> int:
        """A new sequence without tokens (behind a prefix, if given); its number."""
        if prefix is not None and prefix.pages is None:
            raise ValueError("the prefix was dropped")
        self.next += 1
        self.sequences[self.next] = _Sequence(prefix)
        if prefix is not None:
            prefix.users += 1
        return self.next

    def length(self, seq: int) -> int:
        """Tokens of a sequence, its prefix's among them."""
        s = self.sequences[seq]
        return s.length + (s.prefix.length if s.prefix else 0)

    def share(self, seq: int) -> Prefix:
        """Ends a sequence (one without a prefix) and makes its tokens a prefix."""
        if self.sequences[seq].prefix is not None:
            raise ValueError("a sequence behind a prefix cannot become one")
        s = self.sequences.pop(seq)
        return Prefix(s.pages, s.length)

    def drop(self, seq: int) -> None:
        """Ends a sequence; its pages are free again."""
        s = self.sequences.pop(seq)
        self.free += s.pages
        if s.prefix is not None:
            s.prefix.users -= 1

    def drop_prefix(self, prefix: Prefix) -> None:
        """Ends a prefix that no sequence is behind; its pages are free again."""
        if prefix.pages is None:
            raise ValueError("the prefix was dropped before")
        if prefix.users:
            raise ValueError(f"{prefix.users} sequences are behind this prefix")
        self.free += prefix.pages
        prefix.pages, prefix.length = None, 0

    def step(self, new) -> Step:
        """Makes room for new tokens, [(sequence, tokens), ..], each sequence once, all behind the same prefix or none of them
        behind one, and says where they go.  The order is that of their rows."""
        seqs = [self.sequences[i] for i, _ in new]
        if len({i for i, _ in new}) != len(new):
            raise ValueError("a sequence twice in one step")
        if any(n < 0 for _, n in new):
            raise ValueError(f"counts of new tokens {[n for _, n in new]}")
        prefix = seqs[0].prefix if seqs else None
        if any(s.prefix is not prefix for s in seqs):
            raise ValueError("sequences behind different prefixes in one step")
        need = [-(-(s.length + n) // self.size) - len(s.pages) for s, (_, n) in zip(seqs, new)]
        if sum(need) > len(self.free):
            raise RuntimeError(f"{sum(need)} pages are wanted, {len(self.free)} are free")
        slots, positions, offsets = [], [], [0]
        before = prefix.length if prefix else 0
        for s, (_, n), more in zip(seqs, new, need):
            for _ in range(more):
                s.pages.append(self.free.pop())
            for j in range(s.length, s.length + n):
                slots.append(s.pages[j // self.size] * self.size + j % self.size)
                positions.append(before + j)
            s.length += n
            offsets.append(offsets[-1] + n)
        width = max([len(s.pages) for s in seqs] + [1])
        table = [s.pages + [-1] * (width - len(s.pages)) for s in seqs]
        at = lambda v, t: torch.tensor(v, dtype=t, device=self.device)  # noqa: E731
        return Step(at(table, torch.int32).reshape(len(seqs), width), at([s.length for s in seqs], torch.int32), at(offsets, torch.int32),
                    at(slots, torch.int64), at(positions, torch.int64), offsets[-1], max([n for _, n in new] + [0]),
                    at(prefix.pages, torch.int32) if prefix else None, at([prefix.length], torch.int32) if prefix else None)


class Rotary:
    """Rotary positions of the first `rot` elements of each head (binding.nvfp4_rope; scaling as of nvfp4_rope_turns)."""

    def __init__(self, rot: int, base: float = 10000.0, layout: int = B.NVFP4_ROPE_HALVES, magnitude: float = 1.0, device="cuda",
                 **scaling):
        self.turns = B.nvfp4_rope_turns(rot, base, device=device, **scaling)
        self.layout, self.magnitude = layout, magnitude

    def __call__(self, x, positions, out=None):
        """x [tokens, heads, dim] turned, in place or into out."""
        return B.nvfp4_rope(x, positions, self.turns, out, self.magnitude, self.layout)

    def backward(self, d_out, positions, d_x=None):
        """The gradient of x from that of the result, in place or into d_x."""
        return B.nvfp4_rope(d_out, positions, self.turns, d_x, self.magnitude, self.layout, inverse=True)


class KVCache:
    def __init__(self, pages: Pages, heads: int, dim: int = 128, S_k: float = 1.0, S_v: float = 1.0,
                 method: int = B.NVFP4_KV_SWEEP):
        """One layer's pool.  S_k, S_v: the global scales of all keys and values, as numbers or float32 tensors of one
        element (``calibrate`` takes them from samples)."""
        if dim not in (64, 128):
            raise ValueError(f"heads of 64 or 128 elements are wanted, not {dim}")
        self.pages, self.heads, self.dim, self.method = pages, heads, dim, method
        new = lambda *s: torch.zeros(*s, dtype=torch.uint8, device=pages.device)  # noqa: E731
        scale = lambda S: S if isinstance(S, torch.Tensor) else torch.full((1,), float(S), device=pages.device)  # noqa: E731
        self.held = (new(pages.count, heads, 2, pages.size, dim // 2), new(pages.count, heads, 2, dim // 16, pages.size),
                     scale(S_k), scale(S_v))
        self.status = torch.zeros(1, dtype=torch.int32, device=pages.device)

    @staticmethod
    def calibrate(x):
        """The global scale of keys or values like x (bf16 or fp32, on the GPU): amax / (6 * 256)."""
        x = x.contiguous().view(-1)
        S = torch.empty(1, device=x.device)
        ws = torch.empty(B.nvfp4_global_scale_workspace(x.numel()), dtype=torch.uint8, device=x.device)
        B.nvfp4_global_scale(x, 256.0, S, None, ws)
        return S

    def write(self, step: Step, k, v) -> None:
        """A step's new keys and values [tokens, heads, dim] into their slots."""
        B.nvfp4_kv_write(self.held, k, v, step.slots, self.method, self.status)

    def attend(self, step: Step, q, scale: float | None = None, causal: bool = True, out=None, lse=None):
        """Attention of a step's queries [tokens, q_heads, dim] (bf16) over their sequences and the step's prefix."""
        if out is None:
            out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        scale = 1.0 / math.sqrt(self.dim) if scale is None else scale
        batch, width = step.table.shape
        more = 0 if step.prefix is None else step.prefix.numel()
        # a workspace for each call: calls on two streams run at one time
        ws = torch.empty(B.nvfp4_kv_attention_workspace(self.held, q, batch, width, step.max_q, more), dtype=torch.uint8,
                         device=q.device)
        args = (step.table, step.lens, step.offsets, step.max_q, scale, out, causal, lse, ws, self.status)
        if step.prefix is None:
            B.nvfp4_kv_attention(q, self.held, *args)
        else:
            B.nvfp4_kv_attention_prefix(q, self.held, step.prefix, step.prefix_len, *args)
        return out

    def read(self, seq: int, dtype=torch.bfloat16):
        """A sequence's own cached keys and values, each [tokens, heads, dim]."""
        s = self.pages.sequences[seq]
        k, v = (torch.empty(s.length, self.heads, self.dim, dtype=dtype, device=self.pages.device) for _ in range(2))
        table = torch.tensor([s.pages or [-1]], dtype=torch.int32, device=self.pages.device)
        offsets = torch.tensor([0, s.length], dtype=torch.int32, device=self.pages.device)
        B.nvfp4_kv_read(self.held, table, None, offsets, k, v, self.status)
        return k, v


def main(batch: int = 16, length: int = 4096, heads: int = 8, group: int = 4, dim: int = 128) -> None:
    """A batch's prompts and one decoding step: the error of 4-bit attention against fp32, and the times."""
    g = torch.Generator(device="cuda").manual_seed(0)
    draw = lambda n, h: (torch.randn(n, h, dim, device="cuda", generator=g)  # noqa: E731
                         * torch.exp(0.5 * torch.randn(1, h, 1, device="cuda", generator=g))).to(torch.bfloat16)
    pages, rotary = Pages(batch * (-(-(length + 1) // 64)), 64), Rotary(dim, 500000.0)
    k, v = draw(batch * length, heads), draw(batch * length, heads)
    cache = KVCache(pages, heads, dim, KVCache.calibrate(k), KVCache.calibrate(v))
    seqs = [pages.add() for _ in range(batch)]
    step = pages.step([(s, length) for s in seqs])
    rotary(k, step.positions)
    cache.write(step, k, v)
    kn, vn, q = draw(batch, heads), draw(batch, heads), draw(batch, heads * group)
    one = pages.step([(s, 1) for s in seqs])
    rotary(kn, one.positions)
    rotary(q, one.positions)
    cache.write(one, kn, vn)
    out = cache.attend(one, q)
    full = [torch.cat((a.view(batch, length, heads, dim), b[:, None]), 1).float() for a, b in ((k, kn), (v, vn))]
    z = torch.einsum("bhgd,blhd->bhgl", q.float().view(batch, heads, group, dim), full[0]) / math.sqrt(dim)
    want = torch.einsum("bhgl,blhd->bhgd", z.softmax(-1), full[1]).reshape(out.shape)
    err = ((out.float() - want).norm() / want.norm()).item()
    times = []
    for run in (lambda: cache.write(step, k, v), lambda: cache.attend(one, q), lambda: rotary(k, step.positions)):
        for _ in range(3):
            run()
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        for _ in range(20):
            run()
        b.record()
        torch.cuda.synchronize()
        times.append(a.elapsed_time(b) * 50)
    print(f"{batch} sequences of {length} tokens, {heads} key heads of {dim}, {heads * group} query heads: relative error {err:.3f}; "
          f"prompt written in {times[0]:.0f} us, one step of attention {times[1]:.0f} us, keys turned in {times[2]:.0f} us")


if __name__ == "__main__":
    main()
