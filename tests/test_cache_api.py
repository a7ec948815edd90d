"""Refusals and launches of the entry points on rotated rows, bounds of blocks and selected blocks and of a 4-bit
pool, on the CPU (tests/cache_api_driver.cpp): what is refused launches nothing and changes nothing."""

import os
import shutil
import subprocess

import pytest

from conftest import ROOT

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
pytestmark = pytest.mark.skipif(shutil.which(HIPCC) is None, reason="no hipcc")


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    tmp = tmp_path_factory.mktemp("cache_api")
    exe, obj = str(tmp / "cache_api"), str(tmp / "api.o")
    csrc = os.path.join(ROOT, "paper_2503_08461_amd", "csrc")
    subprocess.run([HIPCC, "-x", "hip", "--offload-host-only", "-std=c++17", "-O1", "-fPIC", "-c",
                    os.path.join(ROOT, "tests", "cache_api_driver.cpp"), "-o", obj], check=True)
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", obj, os.path.join(csrc, "fc_plan.cpp"),
                    os.path.join(csrc, "fc_chunk_plan.cpp"), "-o", exe], check=True)

    def run(*args):
        r = subprocess.run([exe, *args], capture_output=True, text=True, timeout=60)
        assert r.returncode == 0, (r.returncode, r.stdout, r.stderr)
        return [ln.split() for ln in r.stdout.splitlines()]
    return run


@pytest.fixture(scope="module")
def calls(driver):
    return driver()


def test_what_is_refused(calls):
    refused = {"create4_small", "compress4", "noalloc4", "var4", "lse4", "window4", "kept4", "mlp4", "quantise4_from8", "quantise4_back",
               "quantise4_other", "rotate_past", "rotate_before", "rotate_far", "rotate_null", "rotate_no_table", "rotate_askew", "rotate_odd",
               "rotate_wide", "rotate_none", "rotate_empty", "rotate_q", "rotate_q_out", "rotate_heads", "rotate_many_heads", "rotate_overlap",
               "rotate_k", "rotate_v", "rotate_layer", "rotate_tables", "rotate_pool", "bounds_null", "bounds_askew", "bounds_layer",
               "bounds_short_table", "bounds_news", "bounds_more", "sparse_none", "sparse_many", "sparse_q", "sparse_out", "sparse_overlap",
               "sparse_heads", "sparse_askew", "sparse_selected", "sparse_bounds", "captured_first", "captured_many"}
    lines = {c[0]: c for c in calls}
    assert refused <= set(lines)
    for name in refused:
        assert lines[name][1] == "-1" and len(lines[name]) == 2, lines[name]
    # (one length's worth of new tokens, and of one request a token too many)
    for c in calls:
        if c[0] not in refused and c[0] not in ("lens", "reads", "kept", "retired"):
            assert c[1] == "0", c


def test_what_is_launched(calls):
    lines = {c[0]: c[2:] for c in calls if c[0] != "reads"}
    assert lines["store4"] == ["store2"] and lines["quantise4"] == ["quantise1"] and lines["quantise8"] == ["quantise0"]
    assert lines["attend4"] == ["attention3x1"] and lines["prefill4"] == ["attention0x1"]
    # positions: those of the cache (101 and 41 tokens, 1 and 33 of them new), or the caller's
    assert lines["rotate"] == ["rotate0_inline:34x0:100:8"] and lines["rotate_last"] == ["rotate0_inline:34x0:999:967"]
    assert lines["rotate4"] == ["rotate2_inline:34x8:100:8"] and lines["rotate8"] == ["rotate1_inline:34x1:100:8"]
    assert lines["rotate_unused"] == ["rotate0_inline:33x0:0"] and lines["rotate_nothing"] == []
    # blocks: 7 + 3, of the new tokens 1 + 3
    assert lines["bounds"] == ["bounds0:10"] and lines["bounds_new"] == ["bounds2:4"] and lines["bounds8"] == ["bounds1:4"]
    assert lines["bounds_nothing"] == [] and lines["sparse_nothing"] == []
    # little to score: one launch for the tokens, which see 101 and 41 tokens, or one 101 and 33 9 to 41
    assert lines["sparse"] == ["selected1_inline:2:6:0,101,0:1,41,1"]
    assert lines["sparse4"] == ["selected3_inline:34:1:0,101,0:1,9,1:1,10,2"] and lines["sparse8"][0].startswith("selected2_inline:34:1:")
    # one long cache: its scores in a launch of their own, 1874 blocks in parts of 64
    assert lines["sparse_long"] == ["select_inline:1:1x30:1874", "attention1x4"]
    assert lines["sparse_apart"] == ["select_inline:3:1x8:500", "attention2x4"] and lines["sparse_rows"][0].startswith("select_inline:2:1x1:6")
    assert lines["captured"] == lines["eager"] == ["select_inline:140:70x140:499", "attention1x4"]
    reads = [[int(x) for x in c[1:]] for c in calls if c[0] == "reads"]
    # 64 blocks of 30000; of 8000 and of 8001 (the last one holds one token), all of 41
    assert reads == [[0, 1024, 1, 0], [0, 1024, 1, 0], [1, 1009, 1, 1], [2, 41, 1, 2]]


def test_scratch_of_captured_calls(calls):
    flags = {c[0]: c[1] for c in calls if c[0] in ("kept", "retired")}
    assert flags == {"kept": "1", "retired": "1"}


def test_calls_within_and_beyond_one_launch(driver):
    lines = driver("limits")
    assert len(lines) == 2 * 2 * 4
    for name, code, *launched in lines:
        assert code == ("-1" if name.endswith("_beyond") else "0") and bool(launched) == name.endswith("_within"), name
