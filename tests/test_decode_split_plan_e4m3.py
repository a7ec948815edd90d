"""How a decode attention over an 8-bit pool takes its heads (csrc/fc_plan.cpp): whole by four or by 16
wavefronts, or cut into segments, every block in exactly one, within the room that the pool has for
their states.  Host code, built with the sanitizers, no GPU."""

import os
import random
import shutil
import subprocess

import pytest

from conftest import ROOT

MAX_SEGMENTS = 16384   # of all heads of a call together


@pytest.mark.skipif(shutil.which("g++") is None, reason="no host compiler")
def test_decode_segments_of_an_8_bit_pool(tmp_path):
    exe = str(tmp_path / "decode_split")
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                    "-static-libasan", "-static-libubsan", os.path.join(ROOT, "tests", "decode_split_e4m3_driver.cpp"),
                    os.path.join(ROOT, "paper_2503_08461_amd", "csrc", "fc_plan.cpp"), "-o", exe], check=True)
    rng = random.Random(8)
    # (case, segments, 16 wavefronts): both sides of the shortest and the longest head that 16 wavefronts take and
    # of as many heads as CUs; twice the smallest segment; no tokens; no memory; room for one segment a head
    fixed = [((1, 4, 256, MAX_SEGMENTS, [240]), 1, 0), ((1, 4, 256, MAX_SEGMENTS, [241]), 1, 1),
             ((1, 4, 256, MAX_SEGMENTS, [2048]), 1, 1), ((1, 4, 256, MAX_SEGMENTS, [2049]), 4, 0),
             ((1, 256, 256, MAX_SEGMENTS, [1024]), 1, 1), ((1, 257, 256, MAX_SEGMENTS, [1008]), 1, 0),
             ((1, 257, 256, MAX_SEGMENTS, [1024, 16]), 2, 0), ((1, 4, 256, MAX_SEGMENTS, [0, 0]), 1, 0),
             ((1, 4, 256, 0, [2049, 5]), 1, 0), ((32, 257, 256, MAX_SEGMENTS, [32768]), 1, 0),
             ((1, 4, 256, 8, [32768]), 2, 0), ((1, 4, 256, 7, [32768]), 1, 0)]
    cases = [f[0] for f in fixed]
    for _ in range(400):
        nl, nh = rng.choice([(1, 4), (1, 32), (2, 12), (32, 32), (80, 64)])
        cases.append((nl, nh, rng.choice([64, 256, 304]), rng.choice([0, 200, MAX_SEGMENTS]),
                      [int(2 ** rng.uniform(0, 15)) - 1 for _ in range(rng.randrange(1, rng.choice([5, 70])))]))
    text = "".join("%d %d %d %d %d %s\n" % (*c[:4], len(c[4]), " ".join(map(str, c[4]))) for c in cases)
    out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout
    got = [tuple(int(x) for x in line.split()) for line in out.splitlines()]
    assert len(got) == len(cases)
    assert [row[1:3] for row in got[:len(fixed)]] == [f[1:] for f in fixed]
    cut = wide = 0
    for (seg, n, sixteen, *rest), (nl, nh, n_cu, room, lens) in zip(got, cases):
        longest = (max(lens) + 15) // 16
        units = len(lens) * nl * nh
        counts = []
        for L in lens:
            blocks, count, at = (L + 15) // 16, rest[0], rest[1:rest[0] + 2]
            rest = rest[count + 2:]
            counts.append(count)
            assert at[0] == 0 and at[-1] == blocks and at == sorted(at)
            sizes = [b - a for a, b in zip(at, at[1:])]
            assert max(sizes) - min(sizes) <= 1 and (n == 1 or min(sizes) > 0 or blocks == 0)
        assert not rest and seg >= 1 and n == max(counts)
        assert sixteen == (units <= n_cu and 16 <= longest <= 128) and not (sixteen and n > 1)
        if n > 1:
            assert 32 <= seg <= longest // 2 and n <= 128 and n * units <= room
        cut += n > 1
        wide += sixteen
    assert cut > 50 and wide > 20
