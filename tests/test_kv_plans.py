"""csrc/kv_plan.h without a GPU: parts cover the keys, clusters are of 1, 2, 4 or 8 blocks, and the shapes of
test_gpu_kv_paths.py take the paths that are written beside them."""
import random

import pytest

import kv_plans as P
import kv_reference as R
import test_gpu_kv_paths as T


def test_shapes_take_their_paths():
    for args, want in T.PATHS:
        assert P.path_of(R.Setting(*args[0], **args[1])) == want, args
    seen = {want for _, want in T.PATHS}
    assert seen >= {(r, j, 0) for r in (8, 16) for j in ("alone", "cluster", "workspace")} | {(r, j, 0) for r in (256, 512) for j in ("alone", "workspace")}
    # the prefix's pass has at least as many rows as a sequence's
    assert seen >= {(r, "merge", q) for r in (8, 16) for q in (8, 16, 256) if q >= r} | {(8, "merge", 512), (256, "workspace", 256), (512, "workspace", 512)}


def sizes(n):
    rng = random.Random(3)
    for _ in range(n):
        heads, dim = rng.choice([1, 2, 5, 8, 64]), rng.choice([64, 128])
        group, batch = rng.choice([1, 2, 4, 7, 8, 16, 40]), int(2 ** rng.uniform(0, 12))
        max_q = int(2 ** rng.uniform(0, 11))
        tokens = min(batch * max_q, 1 << 20)
        yield tokens, batch, min(max_q, tokens), heads * group, heads, dim, int(2 ** rng.uniform(4, 21)), rng.choice([0, 0, 100, 32768])


def test_plans():
    for s in sizes(4000):
        p = P.plan_of(*s)
        if s[0] * s[3] >= 2 ** 31:
            assert not p["fits"] and p["bytes"] == 0
            continue
        assert p["fits"]
        tokens, batch, max_q, q_heads, heads, dim, length, prefix = s
        group = q_heads // heads
        assert p["rows"] * p["tiles"] >= max_q * group and p["rows"] * (p["tiles"] - 1) < max_q * group
        n = max_q * group
        assert p["rows"] in ((8,) if n <= 8 else (16,) if n <= 16 else (256, 512))
        if p["rows"] == 512:                                        # pairs: full ones, long parts
            assert dim == 128 and p["tiles"] * 512 <= n * 1.25 and p["parts"] * 2048 <= length
        assert p["parts"] >= 1 and (p["prefix_parts"] >= 1) == (prefix > 0)
        if p["rows"] < 256:
            assert p["tiles"] == 1
        if not p["through"] or p["merge"]:
            assert p["parts"] in (1, 2, 4, 8)
            assert p["rows"] < 256 or p["parts"] == 1
        parts = 0 if not p["through"] else p["prefix_parts"] if p["merge"] else p["parts"] + p["prefix_parts"]
        assert p["bytes"] >= parts * tokens * q_heads * (dim + 2) * 4 and p["bytes"] % 256 == 0
        assert (p["bytes"] > 0) == p["through"]


def test_parts_cover_the_keys():
    rng = random.Random(4)
    L = P.lib()
    for _ in range(20000):
        length, parts, step = int(2 ** rng.uniform(0, 31)) - 1, rng.choice([1, 2, 4, 8, 19, 152]), rng.choice([64, 128])
        n = L.tokens_of(length, parts, step)
        assert n % step == 0 and n >= step and n * parts >= length
        assert n == step or (n - step) * parts < length                         # no more than needed
        assert L.tokens_of32(length, parts, step) == n


def test_token_numbers_fit_31_bits():
    """The kernels' numbers at the longest tables: where a warp of four starts, its next pages (two tiles of 256 tokens on, 48 within
    one) and a part's tokens as an int, and the tile kernel's key numbers two tiles behind the last."""
    most, L = 2 ** 31 - 2048, P.lib()
    for length in (most, most - 1, most - 63, most - 5000, 2 ** 30 + 1):
        for parts in list(range(1, 9)) + [19, 152, 608, 760]:
            chunk = L.tokens_of32(length, parts, 64)
            assert chunk < 2 ** 31 and chunk * parts >= length
            # parts that join in a cluster all run; others return where they have no keys
            last = parts - 1 if parts <= 8 else (length - 1) // chunk
            assert last * chunk + 3 * 64 + 2 * 256 + 48 < 2 ** 31
            assert length - 1 + 2 * 256 + 48 < 2 ** 31
            tiles = -(-L.tokens_of(length, parts, 128) // 128)
            assert (tiles + 1) * 128 + 127 < 2 ** 31
    p = P.plan_of(1, 1, 1, 4, 1, 128, most)
    assert p["fits"] and p["parts"] * P.lib().tokens_of32(most, p["parts"], 64) >= most


def test_rows_divide_by_a_multiplication():
    """Row r of a block of few rows belongs to query r / group: r (65536 / group + 1) >> 16."""
    for group in range(1, 17):
        for r in range(16):
            assert r * (65536 // group + 1) >> 16 == r // group


def test_largest_sizes():
    big = 2 ** 31 - 1
    for s in ((big, big, 1, 8, 8, 64, 2 ** 30, 0), (big, big, big, 65535, 1, 128, 2 ** 30, 2 ** 30), (1, big, 1, 65535, 65535, 128, 2 ** 30, 0),
              (big, 1, big, 64, 1, 64, 2 ** 30, 0), (2 ** 20, 2 ** 20, 1, 65535, 1, 128, 16, 16)):
        p = P.plan_of(*s)
        assert p["bytes"] >= 0 and p["parts"] >= 1
        assert not p["fits"] or (p["tiles"] * p["parts"] * s[1] < 2 ** 31 and s[0] * s[3] < 2 ** 31)
