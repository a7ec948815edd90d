"""What a pool on a nearly full card has for the states of split caches: as much as chunks of many
tokens can use, else as much as single tokens need, else none, and no call uses more than there is
(tests/segment_memory_driver.cpp, on the CPU)."""

import os
import shutil
import subprocess

import pytest

from conftest import ROOT

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
pytestmark = pytest.mark.skipif(shutil.which(HIPCC) is None, reason="no hipcc")


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    tmp = tmp_path_factory.mktemp("segment_memory")
    exe, obj = str(tmp / "segments"), str(tmp / "api.o")
    csrc = os.path.join(ROOT, "paper_2503_08461_amd", "csrc")
    subprocess.run([HIPCC, "-x", "hip", "--offload-host-only", "-std=c++17", "-O1", "-fPIC", "-c",
                    os.path.join(ROOT, "tests", "segment_memory_driver.cpp"), "-o", obj], check=True)
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", obj, os.path.join(csrc, "fc_plan.cpp"),
                    os.path.join(csrc, "fc_chunk_plan.cpp"), "-o", exe], check=True)
    return exe


# states that the pool's buffer can hold, by the largest allocation in MB
@pytest.mark.parametrize("megabytes,most", [(64, 65536), (12, 16384), (1, 0)])
def test_states_of_split_caches(driver, megabytes, most):
    r = subprocess.run([driver, str(megabytes << 20)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, (r.returncode, r.stdout, r.stderr)
    out = {ln.split()[0]: ln.split()[1:] for ln in r.stdout.splitlines()}
    assert out["decode"][0] == out["chunk"][0] == "0"
    segments = int(out["decode"][1].split(":")[1])
    states, end = int(out["chunk"][1]), int(out["chunk"][2])
    buffer, words = (int(x) for x in out["buffer"])
    if most == 0:
        assert segments == 1 and states == 0 and buffer == 0
        return
    # a decode step's heads are cut as ever: segments of an eighth of a CU's share, (500 + 1875) * 32 / 2048 = 37 blocks
    assert segments == 51
    assert 0 < states <= most and end <= buffer + 4 * words * most
    assert (states > 16384) == (most > 16384)
