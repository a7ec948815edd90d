"""Host planning of positions, bounds, selected blocks and attention over 4-bit rows (csrc/fc_chunk_plan.cpp), under
the host sanitizers.  No GPU."""

import os
import random
import shutil
import subprocess

import pytest

from conftest import ROOT

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="no host compiler")
EINVAL = "-1"


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("cache_plan") / "driver")
    csrc = os.path.join(ROOT, "paper_2503_08461_amd", "csrc")
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-Wall", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                    "-static-libasan", "-static-libubsan", os.path.join(ROOT, "tests", "cache_plan_driver.cpp"),
                    os.path.join(csrc, "fc_chunk_plan.cpp"), "-o", exe], check=True)

    def run(lines):
        out = subprocess.run([exe], input="\n".join(lines) + "\n", capture_output=True, text=True, check=True).stdout
        return [ln.split()[1:] for ln in out.splitlines()]
    return run


def _batch(rows):
    return "%d %s" % (len(rows), " ".join(" ".join(map(str, r)) for r in rows))


def _blocks(n):
    return -(-n // 16)


def _random_batch(rng):
    pairs = []
    for _ in range(rng.choice([1, 1, 2, 5, 40, 120])):
        n = int(2 ** rng.uniform(0, 15))
        pairs.append((n, min(n, rng.choice([0, 1, 1, 1, 3, 30]))))
    return [(n, 1) for n, _ in pairs] if rng.random() < 0.3 else pairs


def test_positions(plan):
    got = plan(["P 100 0 " + _batch([(100, 3, 9), (7, 0, -5), (5, 5, 9)]), "P 99 0 " + _batch([(100, 3, 9)]),
                "P 10 1 " + _batch([(100, 3, 7), (7, 0, -5), (5, 5, 0)]), "P 10 1 " + _batch([(100, 3, 8)]),
                "P 10 1 " + _batch([(100, 3, -1)]), "P 2147483647 1 " + _batch([(9, 9, 2147483638)]),
                "P 2147483647 1 " + _batch([(9, 9, 2147483639)]), "P 2 1 " + _batch([(9, 9, 0)]),
                "P 1 1 " + _batch([(32768, 32768, -2147483648)])])
    assert got == [["0", "0,97", "2,0"], [EINVAL], ["0", "0,7", "2,0"], [EINVAL], [EINVAL], ["0", "0,2147483638"], [EINVAL], [EINVAL], [EINVAL]]


def test_blocks_with_new_tokens(plan):
    got = plan(["B " + _batch([(33, 1), (48, 0), (33, 2), (16, 16), (17, 2), (32768, 32768)]), "B " + _batch([(32768, 32768)] * 8191),
                "B " + _batch([(32768, 32768)] * 8192)])
    assert got[0] == ["0", "2054", "0,2,0", "2,1,1", "3,0,3", "4,0,4", "5,0,6"]
    assert got[1][:2] == ["0", str(8191 * 2048)] and got[2][0] == EINVAL


def test_tokens_parts_and_what_they_read(plan):
    """Every new token reads its own block and at most n_select - 1 others; every block that some token scores is
    in exactly one part of each of the tiles of its request, and tokens know the parts of their tile."""
    rng = random.Random(11)
    lines, cases = [], []
    for _ in range(400):
        pairs = _random_batch(rng)
        heads, group = rng.choice([(1, 1), (8, 4), (32, 1), (2, 33), (3, 64), (40, 1)])
        n_cu, n_select = rng.choice([64, 256]), rng.choice([1, 2, 7, 64, 400, 2048])
        cases.append((pairs, heads, group, n_cu, n_select))
        lines.append("S %d %d %d %d %s" % (heads, group, n_cu, n_select, _batch(pairs)))
    fused = apart = 0
    for (pairs, heads, group, n_cu, n_select), got in zip(cases, plan(lines)):
        code, part, tile, n_units, longest = (int(x) for x in got[:5])
        assert code == 0
        kinds = {k: [[int(v) for v in w[1:].split(",")] for w in got[5:] if w[0] == k] for k in "qta"}
        seen = [(r, n - new + i + 1) for r, (n, new) in enumerate(pairs) for i in range(new)]
        assert [tuple(t[:2]) for t in kinds["t"]] == seen and [t[2] for t in kinds["t"]] == list(range(len(seen)))
        scoring = [_blocks(n) for _, n in seen if _blocks(n) > n_select > 1]
        assert longest == max([nb - 1 for nb in scoring] + [1])
        single = all(new <= 1 for _, new in pairs)
        many = 2 * len(seen) * heads >= n_cu
        read = max([min(_blocks(n), n_select) for _, n in seen] + [0])
        assert (part == 0) == (group <= 32 and read <= (256 if many else 64) and (longest <= 384 or (single and many)))
        if part == 0:
            assert n_units == 0 and not kinds["q"] and not kinds["a"]
            fused += 1
            continue
        assert len(kinds["a"]) == len(seen)
        for row, ((r, n), a) in enumerate(zip(seen, kinds["a"])):
            assert a == [row, n if _blocks(n) <= n_select else (n_select - 1) * 16 + (n - 1) % 16 + 1, 1, row]
        apart += bool(scoring)
        assert part % 16 == 0 and part >= 64 and 1 <= tile and (tile * group <= 64)
        at, first = 0, {}
        for r, new, unit, blocks in kinds["q"]:
            assert new == pairs[r][1] and unit == at and blocks == _blocks(pairs[r][0]) - 1 and blocks >= n_select > 1
            first[r] = unit
            at += -(-new // tile) * -(-blocks // part)
        assert at == n_units and set(first) == {r for r, n in seen if _blocks(pairs[r][0]) > n_select > 1}
        offset = {}
        for (r, n), t in zip(seen, kinds["t"]):
            i = offset.get(r, 0)
            offset[r] = i + 1
            if _blocks(n) > n_select > 1:
                parts = -(-(_blocks(pairs[r][0]) - 1) // part)
                assert t[3:] == [first[r] + i // tile * parts, parts]
    assert fused > 50 and apart > 50
    got = plan(["S 1 1 256 0 1 9 1", "S 1 1 256 2049 1 9 1", "S 256 1 256 2 1 32768 32767", "S 256 1 256 2 1 32768 32768", "S 1 1 256 2 0"])
    assert [g[0] for g in got] == [EINVAL, EINVAL, "0", EINVAL, "0"]


def test_segments_of_4_bit_rows(plan):
    """Units and states do not overlap, states fit, and a head of few rows has at most 64 segments."""
    rng = random.Random(12)
    lines, cases = [], []
    for _ in range(400):
        pairs = _random_batch(rng)
        heads, group = rng.choice([(1, 1), (4, 8), (8, 4), (32, 1), (3, 64), (40, 1)])
        states = rng.choice([0, 100, 65536])
        cases.append((pairs, heads, group, states))
        lines.append("F %d %d 256 %d %s" % (heads, group, states, _batch(pairs)))
    cut = 0
    for (pairs, heads, group, states), got in zip(cases, plan(lines)):
        assert got[0] == "0"
        used, held = 0, []
        few = all(new * group <= 16 for _, new in pairs)
        for tile, text in zip((128, 32), " ".join(got[2:]).split(" | ")):
            words = text.split()
            n_units, seg, n_seg, rows = (int(w) for w in words[:4])
            at = state = 0
            for w in words[4:]:
                r, n, new, unit, state_off = (int(v) for v in w.split(","))
                assert (n, new) == pairs[r] and (new * group <= 32) == (tile == 32) and (unit, state_off) == (at, state)
                mine = max(1, (_blocks(n) + seg // 2) // seg)
                assert mine <= n_seg <= (64 if few else 128)
                at += -(-new * group // tile) * mine
                state += new
                held.append(r)
            assert at == n_units
            if n_seg > 1:
                assert state == rows and seg >= (16 if few else 32)
                used += rows * heads * group * n_seg
                cut += 1
        assert used <= states and sorted(held) == [r for r, p in enumerate(pairs) if p[1]]
    assert cut > 50
