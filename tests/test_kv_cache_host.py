"""kv_cache.Pages without a GPU: which pages and slots tokens get, what a step says, and what it refuses."""
import pytest
import torch

from paper_2606_07618_gb300 import kv_cache as K


def pages(count=10, size=16):
    return K.Pages(count, size, device="cpu")


def test_steps_fill_pages():
    p = pages()
    a, b = p.add(), p.add()
    s = p.step([(a, 20), (b, 1)])
    assert s.tokens == 21 and s.max_q == 20 and s.offsets.tolist() == [0, 20, 21] and s.lens.tolist() == [20, 1]
    assert s.table.dtype == s.lens.dtype == s.offsets.dtype == torch.int32 and s.slots.dtype == s.positions.dtype == torch.int64
    assert s.positions.tolist() == list(range(20)) + [0] and s.prefix is None
    t = p.step([(b, 1), (a, 12)])
    assert t.table.shape == (2, 2) and t.table[0, 1] == -1 and t.lens.tolist() == [2, 32] and t.positions.tolist() == [1] + list(range(20, 32))
    held = {}
    for step, order in ((s, [(a, 0, 20), (b, 0, 1)]), (t, [(b, 1, 1), (a, 20, 12)])):
        slots = iter(step.slots.tolist())
        for row, (q, first, n) in enumerate(order):
            for j in range(first, first + n):
                slot = next(slots)
                assert slot // 16 == step.table[row, j // 16] and slot % 16 == j % 16
                assert held.setdefault(slot, (q, j)) == (q, j)
    assert len(held) == 34 and len(p.free) == 10 - 3
    p.drop(a)
    assert len(p.free) == 9 and p.length(b) == 2


def test_prefix():
    p = pages()
    a = p.add()
    p.step([(a, 40)])
    pre = p.share(a)
    assert pre.length == 40 and a not in p.sequences and len(p.free) == 7
    b, c = p.add(pre), p.add(pre)
    s = p.step([(b, 2), (c, 1)])
    assert s.prefix.tolist() == pre.pages and s.prefix_len.tolist() == [40]
    assert s.positions.tolist() == [40, 41, 40] and s.lens.tolist() == [2, 1] and p.length(b) == 42
    with pytest.raises(ValueError):
        p.share(b)
    with pytest.raises(ValueError):
        p.step([(b, 1), (p.add(), 1)])                             # one behind the prefix, one not
    with pytest.raises(ValueError):
        p.drop_prefix(pre)
    p.drop(b), p.drop(c)
    p.drop_prefix(pre)
    assert len(p.free) == 10


def test_a_dropped_prefix_is_refused():
    """Sequences added behind it would attend without their prompt."""
    p = pages()
    a = p.add()
    p.step([(a, 40)])
    pre = p.share(a)
    p.drop_prefix(pre)
    with pytest.raises(ValueError):
        p.add(pre)
    with pytest.raises(ValueError):
        p.drop_prefix(pre)
    assert len(p.free) == 10 and not p.sequences and pre.users == 0
    b = p.add()
    assert p.step([(b, 3)]).positions.tolist() == [0, 1, 2]


def test_refusals():
    for size in (8, 24, 2048, 0):
        with pytest.raises(ValueError):
            pages(4, size)
    with pytest.raises(ValueError):
        pages(-1)
    p = pages(2)
    a, b = p.add(), p.add()
    with pytest.raises(ValueError):
        p.step([(a, 1), (a, 1)])
    with pytest.raises(ValueError):
        p.step([(a, -1)])
    with pytest.raises(RuntimeError):
        p.step([(a, 17), (b, 16)])                                 # three pages
    assert len(p.free) == 2 and p.length(a) == p.length(b) == 0    # nothing taken
    p.step([(a, 17)])
    with pytest.raises(KeyError):
        p.step([(99, 1)])
    with pytest.raises(ValueError):
        K.KVCache(p, 2, 96)


def test_empty_steps():
    p = pages()
    s = p.step([])
    assert s.tokens == 0 and s.table.shape == (0, 1) and s.offsets.tolist() == [0]
    a = p.add()
    s = p.step([(a, 0)])
    assert s.tokens == 0 and s.max_q == 0 and s.table.tolist() == [[-1]] and s.lens.tolist() == [0]
