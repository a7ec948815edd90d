"""Refusals and launches of the entry points on chunks of new tokens and 8-bit pools, on the CPU
(tests/chunk_api_driver.cpp): what is refused launches nothing and changes nothing."""

import os
import shutil
import subprocess

import pytest

from conftest import ROOT

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
pytestmark = pytest.mark.skipif(shutil.which(HIPCC) is None, reason="no hipcc")


@pytest.fixture(scope="module")
def calls(tmp_path_factory):
    tmp = tmp_path_factory.mktemp("chunk_api")
    exe, obj = str(tmp / "chunk_api"), str(tmp / "api.o")
    csrc = os.path.join(ROOT, "paper_2503_08461_amd", "csrc")
    subprocess.run([HIPCC, "-x", "hip", "--offload-host-only", "-std=c++17", "-O1", "-fPIC", "-c",
                    os.path.join(ROOT, "tests", "chunk_api_driver.cpp"), "-o", obj], check=True)
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", obj, os.path.join(csrc, "fc_plan.cpp"),
                    os.path.join(csrc, "fc_chunk_plan.cpp"), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, (r.returncode, r.stdout, r.stderr)
    return [ln.split() for ln in r.stdout.splitlines()]


def test_what_is_refused(calls):
    refused = {"create8_small", "create_dtype", "compress8", "noalloc8", "var8", "lse8", "window8", "kept8", "mlp8", "weights8",
               "extend_negative", "extend_far", "extend_table", "extend_news", "extend_pool", "store_layer", "store_below",
               "store_null", "store_no_data", "store_odd_stride", "store_backwards", "store_askew", "store_wide", "store_tall",
               "store_too_many", "store_short_table", "attend_heads", "attend_few_heads", "attend_large_group", "attend_window",
               "attend_negative_window", "attend_lse_askew", "attend_layer", "attend_q", "attend_out", "attend_overlap",
               "attend_broadcast_out", "attend_close", "attend_split", "prefill_k", "prefill_v", "prefill_lens", "prefill_beyond",
               "quantise_back", "quantise_other", "quantise_table", "quantise_null"}
    lines = {c[0]: c for c in calls if c[0] != "lens"}
    assert refused <= set(lines)
    for name in refused:
        assert lines[name][1:] == ["-1"], lines[name]
    assert lines["extend_full"][1:] == ["-2"]
    for name, c in lines.items():
        if name not in refused and name != "extend_full":
            assert c[1] == "0", c
    # lengths after the appends, the extension (two blocks of 64: 41 + 30 tokens) and what was refused
    assert [c[1:] for c in calls if c[0] == "lens"] == [["101", "41"], ["101", "71", "free", "62"], ["101", "71", "free", "62"]]


def test_what_is_launched(calls):
    got = {c[0]: c[2:] for c in calls if c[0] != "lens"}
    assert got["append8"] == ["append_inline"] and got["decode8"] == ["attention_inline:1"]
    assert got["extend"] == ["extend_inline"] and got["extend_none"] == []
    assert got["store"] == ["store_inline:34"] == got["store_broadcast"] and got["store8"] == ["store8_inline:34"]
    assert got["store_nothing"] == []
    # a request of 66 rows to a head and one of 2
    assert got["attend"] == ["attention1_inline:1x1:1x1"] and got["attend8"] == ["attention2_inline:1x1:1x1"]
    assert got["attend_group"] == ["attention1_inline:2x1:0x1"]
    assert got["attend_broadcast_q"] == got["attend_head_major"] == got["attend"]
    assert got["attend_split_table"][0].startswith("attention1_inline:0x1:1x") and int(got["attend_split_table"][0].rsplit("x", 1)[1]) > 1
    assert got["prefill"] == ["attention0_inline:1x1:1x1"] and got["prefill_none"] == []
    assert got["quantise"] == ["quantise:8"] and got["quantise_off"] == []
    assert got["many_store"] == ["copy", "store:150"] and got["many_attend"] == ["copy", "attention1:0x1:150x1"]
    assert got["many_store_captured"] == ["upload", "upload", "store:150"]
    assert got["many_attend_captured"] == ["upload", "upload", "attention1:0x1:150x1"]
