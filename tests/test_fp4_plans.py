"""csrc/fp4_plan.h without a GPU: the shapes of test_gpu_fp4_paths.py take the paths that are written beside them, and
between them every path that any size takes."""
import pytest

import fp4_plans as P
import test_gpu_fp4_paths as T


def path(p):
    return (p["tokens"], p["split"], p["whole"]) if p["few"] else (p["width"], p["split"], p["walks"])


@pytest.mark.parametrize("fmt", [P.NV, P.MX])
def test_shapes_take_their_paths(fmt):
    for s, want in T.MATMUL:
        assert path(P.matmul(fmt, *s)) == path(P.matmul(fmt, *s, f32=True)) == want, s
    for s, want in T.GATED:
        assert path(P.gated(fmt, *s)) == want, s
    for s, *want in T.MATMUL_GRADS:
        assert [path(p) for p in P.matmul_grads(*s)] == want, s
    for s, *want in T.GATED_GRADS:
        assert [path(p) for p in P.gated_grads(fmt, *s)] == want, s


def test_parts_of_k_are_split_and_walked():
    """NVFP4's d_x, whose K has two parts: of each width, alone and over several tiles, and over two and four pairs, each
    of which then has one part only."""
    xs = [P.gated_grads(P.NV, *s)[1] for s, *_ in T.GATED_GRADS]
    assert {path(p) for p in xs} >= {(128, 1, True), (224, 1, True), (256, 1, True), (128, 2, False), (256, 2, False),
                                     (128, 4, False), (256, 4, False), (256, 1, False)}
    for p in xs:
        assert p["part"] * 2 == p["stages"] and (p["split"] == 1 or p["stages"] % p["split"] == 0)


# small sizes that the paths of large and small calls share: covered by test_gpu_fp4.py's shapes
ELSEWHERE = {(16, 1, False), (16, 2, False), (16, 8, False), (32, 8, False), (128, 1, False), (256, 1, False), (128, 4, False),
             (256, 4, False)}


def sizes():
    for t in (1, 17, 33, 70, 256, 500, 1000, 2048, 4096, 9000):
        for n in list(range(32, 2048, 160)) + list(range(2048, 24000, 1376)):
            yield t, n


@pytest.mark.parametrize("fmt", [P.NV, P.MX])
def test_no_other_path_is_taken(fmt):
    ks = (32, 256, 800, 2048, 4096, 8192, 12288, 16384, 40960)
    mm, gated, grad = (set(ELSEWHERE) for _ in range(3))
    mm |= {w for _, w in T.MATMUL}
    gated |= {w for _, w in T.GATED}
    grad |= {w for _, *ws in T.MATMUL_GRADS + T.GATED_GRADS for w in ws}
    for t, n in sizes():
        for k in ks:
            for f32 in (False, True):
                assert path(P.matmul(fmt, t, n, k, f32)) in mm, (t, n, k)
            assert path(P.gated(fmt, t, n, k)) in gated, (t, n, k)
            assert path(P.plan_of(fmt, P.GRAD, t, n, k)) in {(256, s, w) for s in (1, 2, 4) for w in (False, True)}
            for ld in (64, 72):
                assert path(P.plan_of(P.BF16, P.PLAIN, t, n, k, ldq=ld)) in grad, (t, n, k, ld)


@pytest.mark.parametrize("kind", [P.NV, P.MX, P.BF16])
def test_what_a_plan_keeps_to(kind):
    """Each pair has stages to add, clusters find room, and tiles are of the widths that their loads allow."""
    for t, n in sizes():
        for k in (32, 1024, 8192, 65536):
            p = P.plan_of(kind, P.PLAIN, t, n, k, ldq=64)
            assert p["split"] <= max(1, p["stages"])
            if not p["few"]:
                assert p["width"] in ((128, 224, 256) if kind == P.BF16 else (128, 256))
                assert p["split"] == 1 or (p["stages"] >= 8 * p["split"] and 2 * p["split"] * p["tiles"] <= P.SMS
                                           and p["width"] % (32 * p["split"]) == 0)
