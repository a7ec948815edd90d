"""Scratch memory of the attention over selected blocks, on the CPU (tests/sparse_memory_driver.cpp): no more than
include/fastcache.h says, and a call whose memory is not there returns FC_EDEVICE before anything is queued and leaves
the pool as it was."""

import os
import random
import shutil
import subprocess

import pytest

from conftest import ROOT

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
pytestmark = pytest.mark.skipif(shutil.which(HIPCC) is None, reason="no hipcc")


@pytest.fixture(scope="module")
def run(tmp_path_factory):
    tmp = tmp_path_factory.mktemp("sparse_memory")
    exe, obj = str(tmp / "sparse_memory"), str(tmp / "api.o")
    csrc = os.path.join(ROOT, "paper_2503_08461_amd", "csrc")
    subprocess.run([HIPCC, "-x", "hip", "--offload-host-only", "-std=c++17", "-O1", "-fPIC", "-c",
                    os.path.join(ROOT, "tests", "sparse_memory_driver.cpp"), "-o", obj], check=True)
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", obj, os.path.join(csrc, "fc_plan.cpp"),
                    os.path.join(csrc, "fc_chunk_plan.cpp"), "-o", exe], check=True)

    def go(lines=()):
        r = subprocess.run([exe], input="\n".join(lines) + "\n", capture_output=True, text=True, timeout=60)
        assert r.returncode == 0, (r.returncode, r.stdout, r.stderr)
        return [ln.split() for ln in r.stdout.splitlines()]
    return go


def _most(heads, tokens, n_select, blocks):
    """What the header says, to whole 4 KB."""
    need = tokens * heads * 4 * (n_select + blocks + blocks // 64 + 1)
    return -(-(need + need // 8) // 4096) * 4096


def test_no_more_than_documented(run):
    rng = random.Random(4)
    lines, cases = [], []
    for _ in range(200):
        pairs = []
        for _ in range(rng.choice([1, 2, 7, 40])):
            n = int(2 ** rng.uniform(0, 15))
            pairs.append((n, min(n, rng.choice([0, 1, 1, 5, 200]))))
        heads, group, n_select = rng.choice([1, 8, 32]), rng.choice([1, 4, 40, 64]), rng.choice([1, 2, 64, 300])
        cases.append((pairs, heads, n_select))
        lines.append("%d %d %d %d %s" % (heads, group, n_select, len(pairs), " ".join("%d %d" % p for p in pairs)))
    taken = 0
    got = [ln for ln in run(lines) if ln[0] == "batch"]
    assert len(got) == len(cases)
    for (pairs, heads, n_select), (_, code, size) in zip(cases, got):
        assert code == "0"
        tokens, blocks = sum(n for _, n in pairs), max(-(-n // 16) for n, _ in pairs)
        assert int(size) <= _most(heads, tokens, n_select, blocks)
        taken += int(size) > 0.8 * _most(heads, tokens, n_select, blocks)
    assert taken > 10


def test_memory_that_is_not_there(run):
    lines = {ln[0]: ln[1:] for ln in run() if ln[0] != "batch"}
    assert lines["few"] == ["0", "select", "attention"] == lines["few_after"]
    assert lines["chunk_without"] == ["-3"]
    assert lines["chunk"][0] == "0" and lines["chunk"][-2:] == ["select", "attention"]
