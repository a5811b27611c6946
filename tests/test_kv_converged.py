"""The attention kernels' source: instructions that all lanes of a warp execute together (.sync.aligned) are not reached by lanes that
went different ways.  No lane leaves a pass of a loop that holds one on its own, and where lanes took different branches a
__syncwarp() stands before the next one."""
import os
import re

import pytest

from conftest import ROOT

CSRC = os.path.join(ROOT, "paper_2606_07618_gb300", "csrc")
ALIGNED = r"\b(tmem_ld16|tmem_ld32|tmem_st16|tmem_wait_ld|tmem_wait_st|wait_ld32|mma16|mma16_first|transpose8x8|cluster_arrive|cluster_wait)\b\s*(<[^<>]*>)?\("
# answers that all lanes of a warp share
UNIFORM = r"mbar_wait_warp|wait_for|!ok"


def source(name):
    s = open(os.path.join(CSRC, name)).read()
    return re.sub(r"//[^\n]*", lambda m: " " * len(m.group()), s)


def closing(s, at, pair):
    depth = 0
    for i in range(at, len(s)):
        depth += (s[i] == pair[0]) - (s[i] == pair[1])
        if depth == 0:
            return i
    raise AssertionError("unbalanced")


def loops(s):
    """(head, body, position) of every loop with a body in braces."""
    for m in re.finditer(r"\b(for|while)\s*\(", s):
        end = closing(s, m.end() - 1, "()")
        rest = re.match(r"\s*\{", s[end + 1:])
        if rest:
            at = end + rest.end()
            yield s[m.start():end + 1], s[at:closing(s, at, "{}") + 1], m.start()


def at_fault(s):
    """Statements by which some lanes may leave a pass that executes an aligned instruction."""
    found = []
    for head, body, at in loops(s):
        if not re.search(ALIGNED, body):
            continue
        for m in re.finditer(r"\b(continue|break|return)\b", body):
            inner = [b for h, b, _ in loops(body[1:]) if body.find(b) <= m.start() < body.find(b) + len(b)]
            if inner and not any(re.search(ALIGNED, b) for b in inner):
                continue                                           # of a loop inside, which executes none
            condition = body[max(body.rfind("if (", 0, m.start()), 0):m.start()]
            if m.group(1) == "continue" or not re.search(UNIFORM, condition):
                found.append((s[:at].count("\n") + body[:m.start()].count("\n") + 1, m.group(1)))
    return found


@pytest.mark.parametrize("name", ["kv_attention.cu", "kv_attention_tile.cu"])
def test_no_lane_leaves_a_pass(name):
    assert at_fault(source(name)) == []


def test_the_reading_finds_it():
    bad = "for (int c = 0; c < D; c += 16) { tmem_ld16(to + c, o); if (!valid) continue; store(o); }"
    good = "for (int c = 0; c < D; c += 16) { if (!mbar_wait_warp(b, 0)) { ok = false; break; } tmem_ld16(to, o); if (valid) store(o); }"
    nested = "for (int c = 0; c < D; c++) { tmem_ld16(to, o); for (int i = 0; i < 4; i++) { if (i > n) continue; store(o); } }"
    assert at_fault(bad) and not at_fault(good) and not at_fault(nested)


# (file, code after which lanes may have gone different ways, the aligned instruction that comes next)
MEETINGS = [
    ("kv_attention_tile.cu", "if (!whole) {", "float tops[4]"),
    ("kv_attention_tile.cu", "const float alpha =", "tmem_ld16(to + c, o)"),
    ("kv_attention_tile.cu", "if (grown) m", "tmem_st16(ts"),
    ("kv_attention_tile.cu", "const bool valid = row < rows;", "tmem_ld16(to + c, o)"),
    ("kv_attention_tile.cu", "d[i] = (uint16_t)(w[i / 2] >> (16 * (i & 1)));", "a NaN sum shows in both"),
    ("kv_attention.cu", "for (int k0 = start;", "mma16_first(sc"),
    ("kv_attention.cu", "const float alpha =", "transpose8x8(f16x2"),
    ("kv_attention.cu", "if (!vv_ok ||", "mma16(o[nt]"),
    ("kv_attention.cu", "*reinterpret_cast<float4*>(s_o + place(0, r, q)) = v;", "cluster_arrive();"),
    ("kv_attention.cu", "write_row<D, false>(p, 0,", "cluster_arrive();"),
]


@pytest.mark.parametrize("name,branch,then", MEETINGS)
def test_lanes_meet_again(name, branch, then):
    s = open(os.path.join(CSRC, name)).read()
    at = s.index(branch)
    assert "__syncwarp();" in s[at:s.index(then, at)]
