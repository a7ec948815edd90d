"""Host planning of the calls on chunks of new tokens (csrc/fc_chunk_plan.cpp), under the host
sanitizers: refusals, block hand-out, work units and segments.  No GPU."""

import os
import random
import shutil
import subprocess

import pytest

from conftest import ROOT

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="no host compiler")
EINVAL, ENOMEM = -1, -2


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("chunk_plan") / "driver")
    csrc = os.path.join(ROOT, "paper_2503_08461_amd", "csrc")
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-Wall", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                    "-static-libasan", "-static-libubsan", os.path.join(ROOT, "tests", "chunk_plan_driver.cpp"),
                    os.path.join(csrc, "fc_chunk_plan.cpp"), "-o", exe], check=True)

    def run(lines):
        out = subprocess.run([exe], input="\n".join(lines) + "\n", capture_output=True, text=True, check=True).stdout
        return [ln.split()[1:] for ln in out.splitlines()]
    return run


def _batch(pairs):
    return "%d %s" % (len(pairs), " ".join("%d %d" % p for p in pairs))


def test_extend(plan):
    got = plan(["E 10 4 " + _batch([(0, 17), (16, 0), (15, 1), (16, 1), (33, 31)]),
                "E 3 4 " + _batch([(0, 17), (16, 16), (15, 1), (16, 1)]), "E 9 9 0",
                "E 9 2 " + _batch([(32, 1)]), "E 9 2 " + _batch([(-1, 1)]), "E 9 2 " + _batch([(1, -1)]),
                "E 9999 9999 " + _batch([(32768, 0)]), "E 9999 9999 " + _batch([(32768, 1)]),
                "E 9999 9999 " + _batch([(1, 2147483647)]), "E 9 0 " + _batch([(1, 1)]), "E 9 9 -1"])
    assert got[0] == ["0", "4", "0,0,2,0", "3,1,1,2", "4,3,1,3"]
    assert got[1][0] == str(ENOMEM) and got[2] == ["0", "0"]
    assert [g[0] for g in got[3:]] == [str(c) for c in (EINVAL, EINVAL, EINVAL, 0, EINVAL, EINVAL, EINVAL, EINVAL)]


def test_rows_of_a_batch(plan):
    got = plan(["C 4 " + _batch([(5, 5), (64, 0), (64, 1), (0, 0), (20, 7)]), "C -1 " + _batch([(5, 9), (0, 9), (7, 9)]),
                "C 4 " + _batch([(65, 1)]), "C 4 " + _batch([(3, 4)]), "C 4 " + _batch([(3, -1)]), "C 4 " + _batch([(-3, 0)]),
                "C 4096 " + _batch([(32769, 1)]), "C 0 " + _batch([(1, 1)]), "C 4 -2", "C 4 0"])
    assert got[0] == ["0", "0,5,5,0", "2,64,1,5", "4,20,7,6"]
    assert got[1] == ["0", "0,5,5,0", "2,7,7,5"]
    assert [g[0] for g in got[2:]] == [str(c) for c in (EINVAL,) * 7 + (0,)]


def test_blocks_to_quantise(plan):
    got = plan(["Q 4 3 " + _batch([(33, 1), (48, 0), (0, 1), (48, 1)]), "Q 4 2 " + _batch([(33, 1)]), "Q 2 4 " + _batch([(33, 1)]),
                "Q 4 4 " + _batch([(-1, 1)]), "Q 4 4 " + _batch([(32769, 1)])])
    assert got == [["0", "6"]] + [[str(EINVAL)]] * 4


def test_units_and_segments(plan):
    """Every row tile of every request has its segments, units and states do not overlap, states fit."""
    rng = random.Random(5)
    lines, cases = [], []
    for _ in range(300):
        heads, group = rng.choice([(1, 1), (4, 8), (8, 4), (32, 1), (3, 64), (40, 1)])
        n = rng.choice([1, 1, 2, 5, 40, 200])
        pairs = []
        for _ in range(n):
            L = int(2 ** rng.uniform(0, 15))
            pairs.append((L, min(L, rng.choice([0, 1, 1, 3, int(2 ** rng.uniform(0, 11))]))))
        states = rng.choice([0, 100, 65536])
        cases.append((heads, group, pairs, states))
        lines.append("A 2 %d %d %d 1 %d %s" % (heads, group, rng.choice([64, 256]), states, _batch(pairs)))
    split = 0
    for (heads, group, pairs, states), got in zip(cases, plan(lines)):
        assert got[0] == "0"
        kinds = " ".join(got[2:]).split(" | ")
        assert len(kinds) == 2
        used, seen = 0, []
        for tile, text in zip((128, 32), kinds):
            words = text.split()
            n_units, seg, n_seg, rows = (int(w) for w in words[:4])
            at = state = 0
            last = 1 << 30
            for w in words[4:]:
                r, L, n_new, row_off, unit, state_off = (int(v) for v in w.split(","))
                assert (L, n_new) == pairs[r] and row_off == sum(p[1] for p in pairs[:r]) and L <= last
                assert (n_new * group <= 32) == (tile == 32) and unit == at and state_off == state
                last, blocks = L, -(-L // 16)
                mine = max(1, (blocks + seg // 2) // seg)
                assert mine <= n_seg <= 128
                at += -(-n_new * group // tile) * mine
                state += n_new
                seen.append(r)
            assert at == n_units
            if n_seg > 1:
                assert state == rows and seg >= 32
                used += rows * heads * group * n_seg
                split += 1
        assert used <= states and sorted(seen) == [r for r, p in enumerate(pairs) if p[1]]
    assert split > 50


def test_too_large_for_one_launch(plan):
    got = plan(["A 1 65536 64 256 1 0 " + _batch([(32768, 32768)] * 2)])
    assert got[0][0] == str(EINVAL)
