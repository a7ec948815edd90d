"""Calls on more requests than fit a kernel's arguments, captured into a graph: what a replay writes
and reads stays the pool's however large later calls are, and a capture that would have to allocate is
refused.  On the CPU the memory's bookkeeping (tests/captured_requests_driver.cpp)."""

import os
import shutil
import subprocess

import numpy as np
import pytest

from conftest import ROOT

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


@pytest.mark.skipif(shutil.which(HIPCC) is None, reason="no hipcc")
def test_descriptors_of_captured_calls_stay(tmp_path):
    exe, obj = str(tmp_path / "captured"), str(tmp_path / "api.o")
    csrc = os.path.join(ROOT, "paper_2503_08461_amd", "csrc")
    subprocess.run([HIPCC, "-x", "hip", "--offload-host-only", "-std=c++17", "-O1", "-fPIC", "-c",
                    os.path.join(ROOT, "tests", "captured_requests_driver.cpp"), "-o", obj], check=True)
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", obj, os.path.join(csrc, "fc_plan.cpp"),
                    os.path.join(csrc, "fc_chunk_plan.cpp"), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, (r.returncode, r.stdout, r.stderr)
    lines = [ln.split() for ln in r.stdout.splitlines()]
    code = {x[0]: x[1] for x in lines if x[0] not in ("kept", "same", "grown")}
    refused = {"captured_first", "captured_more"}
    assert {n for n, c in code.items() if c != "0"} == refused and all(code[n] == "-1" for n in refused)
    assert [x[1] for x in lines if x[0] in ("same", "grown")] == ["1", "1"]
    # (a buffer has room for twice the requests that it was made for: the last call fits the one of 50 000)
    assert [int(x[1]) for x in lines if x[0] == "kept"] == [0, 0, 0, 0, 0, 1, 1, 1, 1]


@pytest.mark.gpu
@pytest.mark.parametrize("what", ["chunk", "decode"])
def test_replays_after_larger_calls(what):
    """200 requests captured, then an eager call on 1500: every replay is the eager result."""
    import torch
    from paper_2503_08461_amd import fastcache as fc
    dev, n, many, heads, d, blocks = "cuda", 200, 1500, 2, 64, 400
    torch.manual_seed(7)
    kv = torch.randn((1, blocks, 2, heads, 16, d), device=dev).half()
    pool = fc.fc_pool_create(kv, blocks, 1, heads, d)
    try:
        table = torch.randint(0, blocks, (many, 3), dtype=torch.int32, device=dev)
        lens = np.random.default_rng(7).integers(1, 49, many).astype(np.int32)
        ones = np.ones(many, np.int32)
        q = torch.randn((many, 1, heads, d), device=dev).half()

        def step(m, out):
            if what == "decode":
                return fc.fc_decode_attention(pool, table[:m], lens[:m], q[:m], out=out)
            return fc.fc_chunk_attention(pool, 0, table[:m], lens[:m], ones[:m], q[:m, 0], out=out)

        out = step(n, None)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(n, out)
        everyone = step(many, None)
        torch.cuda.synchronize()
        for _ in range(3):
            q.copy_(torch.randn(q.shape, device=dev).half())
            out.zero_()
            step(many, everyone)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, step(n, None))
    finally:
        fc.fc_pool_destroy(pool)
