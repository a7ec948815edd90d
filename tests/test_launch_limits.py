"""A launch has fewer than 2^32 threads, 2^24 workgroups of 256: calls that would need more are refused
before anything is launched or changed (tests/launch_limits_driver.cpp, on the CPU)."""

import os
import shutil
import subprocess

import pytest

from conftest import ROOT

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


@pytest.mark.skipif(shutil.which(HIPCC) is None, reason="no hipcc")
def test_calls_within_and_beyond_one_launch(tmp_path):
    exe, obj = str(tmp_path / "limits"), str(tmp_path / "api.o")
    csrc = os.path.join(ROOT, "paper_2503_08461_amd", "csrc")
    subprocess.run([HIPCC, "-x", "hip", "--offload-host-only", "-std=c++17", "-O1", "-fPIC", "-c",
                    os.path.join(ROOT, "tests", "launch_limits_driver.cpp"), "-o", obj], check=True)
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", obj, os.path.join(csrc, "fc_plan.cpp"),
                    os.path.join(csrc, "fc_chunk_plan.cpp"), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, (r.returncode, r.stdout, r.stderr)
    out = {ln.split()[0]: ln.split()[1:] for ln in r.stdout.splitlines()}
    for call in ("store", "store8", "prefill", "chunk", "quantise", "append", "append8", "decode", "decode8", "kept"):
        assert out[call + "_within"][0] == "0" and len(out[call + "_within"]) > 1, call
        assert out[call + "_beyond"] == ["-1"], call
    assert out["append_within_left"] == ["21"] and out["append_beyond_left"] == ["20"]
