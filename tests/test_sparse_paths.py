"""The cases of test_gpu_sparse_apart.py take the launches that they are for, on a card of 256 compute units: a changed
rule must not leave them without their subject.  No GPU."""

import os
import shutil
import subprocess

import pytest

from conftest import ROOT
from test_gpu_sparse_apart import APART, FEW_ROWS

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="no host compiler")


@pytest.fixture(scope="module")
def paths(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("sparse_paths") / "driver")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", os.path.join(ROOT, "tests", "sparse_path_driver.cpp"),
                    os.path.join(ROOT, "paper_2503_08461_amd", "csrc", "fc_chunk_plan.cpp"), "-o", exe], check=True)

    def run(head, lens, news):
        line = "%s %d %s\n" % (head, len(lens), " ".join("%d %d" % x for x in zip(lens, news)))
        return [int(x) for x in subprocess.run([exe], input=line, capture_output=True, text=True, check=True).stdout.split()]
    return run


def test_scores_of_several_heads_are_made_apart(paths):
    seen = []
    for lens, news, heads, group, _, n_select in APART:
        assert heads > 1
        parts, tiles, segments, segments4 = paths("S %d %d %d" % (heads, group, n_select), lens, news)
        assert parts > 0, (lens, news)                  # (0: one launch for everything)
        seen.append((parts, tiles, segments, segments4))
    # over several parts, several tiles of tokens, with results joined from segments in either way, and whole ones
    assert sum(s[0] > 1 for s in seen) >= 3 and max(s[0] for s in seen) >= 7 and max(s[1] for s in seen) > 1
    assert sum(s[2] > 1 for s in seen) >= 2 and sum(s[3] > 1 for s in seen) >= 2 and min(s[2] for s in seen) == 1


def test_few_rows_of_several_heads_are_cut(paths):
    for lens, news, heads, group, _ in FEW_ROWS:
        tall, flat, segments, rows = paths("C %d %d" % (heads, group), lens, news)
        assert heads > 1 and group > 1 and tall == 0 and segments > 1 and rows <= 16 and flat > len(lens)
