"""Compressions and log-sum-exps captured into a graph: the memory that their replays use stays the
pool's when a later call needs more, and a capture that would have to allocate is refused with nothing
queued or changed.  On the CPU the memory's bookkeeping (tests/captured_scratch_driver.cpp)."""

import os
import shutil
import subprocess

import numpy as np
import pytest

from conftest import ROOT

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


@pytest.fixture(scope="module")
def steps(tmp_path_factory):
    if shutil.which(HIPCC) is None:
        pytest.skip("no hipcc")
    tmp = tmp_path_factory.mktemp("captured_scratch")
    exe, obj = str(tmp / "captured"), str(tmp / "api.o")
    subprocess.run([HIPCC, "-x", "hip", "--offload-host-only", "-std=c++17", "-O1", "-fPIC", "-c",
                    os.path.join(ROOT, "tests", "captured_scratch_driver.cpp"), "-o", obj], check=True)
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", obj, os.path.join(ROOT, "paper_2503_08461_amd", "csrc", "fc_plan.cpp"),
                    "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, (r.returncode, r.stdout, r.stderr)
    return {ln.split()[0]: ln.split()[1:] for ln in r.stdout.splitlines()}


def _counts(steps, name):
    """(code, device buffers made, freed)"""
    return tuple(int(x) for x in steps[name][:3])


@pytest.mark.parametrize("what", ["lse_first", "fused_first", "fused_more", "separate_first", "mlp_first", "weights_captured"])
def test_a_capture_that_would_have_to_allocate(steps, what):
    assert _counts(steps, what) == (-1, 0, 0) and steps[what][3:] == []
    if what != "weights_captured":
        assert steps[what + "_left"] == ["1", "1"]


@pytest.mark.parametrize("what", ["checked_first", "checked_mlp", "checked_free"])
def test_a_capture_with_ownership_checks(steps, what):
    """The checks wait for the device: refused before anything is queued."""
    assert _counts(steps, what) == (-1, 0, 0) and steps[what][3:] == [] and steps[what + "_left"] == ["1", "1"]


@pytest.mark.parametrize("what", ["lse_captured", "fused_noalloc", "fused_captured", "split_captured", "separate_captured",
                                  "mlp_captured"])
def test_a_capture_that_finds_what_it_needs(steps, what):
    assert _counts(steps, what) == (0, 0, 0) and steps[what][3:]


@pytest.mark.parametrize("what,buffers", [("lse", 1), ("fused", 2), ("split", 2), ("separate", 4), ("mlp", 2)])
def test_what_a_replay_uses_stays(steps, what, buffers):
    """The first call that needs more makes new buffers and frees none; with the pool all go."""
    assert _counts(steps, what + "_grows") == (0, buffers, 0)
    assert steps[what + "_end"] == ["0"]


@pytest.mark.parametrize("what,made,freed", [("lse", 1, 1), ("fused", 2, 2), ("split", 3, 2)])
def test_what_no_graph_uses_goes(steps, what, made, freed):
    """(split: scores and kept lists were replaced before, the block ids are not until now)"""
    assert _counts(steps, what + "_grows_again") == (0, made, freed)


def test_weights_of_a_captured_call_stay(steps):
    assert _counts(steps, "weights") == (0, 6, 0) and _counts(steps, "weights_replaced") == (0, 6, 6)
    assert _counts(steps, "weights_kept") == (0, 6, 0) and _counts(steps, "weights_replaced_again") == (0, 6, 6)


@pytest.mark.gpu
@pytest.mark.parametrize("what", ["window_lse", "compress", "mlp"])
def test_replays_after_larger_calls(what):
    """40 requests captured, then an eager call on 1500 (and other weights): every replay leaves what
    the eager call on the 40 left."""
    import torch
    from paper_2503_08461_amd import fastcache as fc
    dev, n, many, heads, d, window = torch.device("cuda:0"), 40, 1500, 2, 64, 16
    blocks = many * 9 + 16
    torch.manual_seed(3)
    kv = torch.randn((1, blocks, 2, heads, 16, d), device=dev).half()
    pool = fc.fc_pool_create(kv, blocks, 1, heads, d)
    try:
        lens = np.random.default_rng(3).integers(40, 97, many).astype(np.int32)
        budgets = np.full(many, 33, np.int32)
        knorm, zeros = np.full(many, fc.FC_METHOD_KNORM, np.int32), np.zeros(many, np.int32)
        q = torch.randn((many, 1, heads, window, d), device=dev).half()
        lse = torch.zeros((many, 1, heads, window), device=dev)

        def set_weights(seed):
            g = torch.Generator(device=dev).manual_seed(seed)
            w1, w2 = ([torch.randn(s, generator=g, device=dev).half() / 8 for _ in range(2)] for s in ((128, 2 * d), (d, 128)))
            b1, b2 = ([torch.randn(s, generator=g, device=dev) / 8 for _ in range(2)] for s in (128, d))
            fc.fc_mlp_set_weights(pool, 2, w1, b1, w2, b2)

        table = torch.full((many, 6), -1, dtype=torch.int32, device=dev)
        start = np.zeros(many, np.int32)
        fc.fc_extend_batch(pool, table, start, lens)
        stack, top = fc.fc_pool_export_state(pool)
        stack0, kv0, table0 = torch.from_numpy(stack).to(dev), kv.clone(), table.clone()

        def rewind():
            fc.fc_pool_import_state_dev(pool, stack0, top)
            kv.copy_(kv0)
            table.copy_(table0)
            lse.zero_()
            torch.cuda.synchronize()

        def call(m):
            now = lens[:m].copy()
            if what == "window_lse":
                fc.fc_window_lse(pool, table[:m], now, q[:m], window, None, lse[:m])
            elif what == "compress":
                fc.fc_compress_batch(pool, table[:m], now, None, window, knorm[:m], budgets[:m])
            else:
                fc.fc_compress_batch_mlp(pool, table[:m], now, zeros[:m], now.copy(), None)

        def state():
            torch.cuda.synchronize()
            return [kv.view(torch.int16).clone(), table.clone(), torch.from_numpy(fc.fc_pool_export_state(pool)[0]), lse.clone()]

        if what == "mlp":
            set_weights(1)
        rewind()
        call(n)
        want = state()
        assert not all(torch.equal(a, b) for a, b in zip(want, (kv0.view(torch.int16), table0, stack0.cpu(), torch.zeros_like(lse))))
        rewind()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call(n)
        for i in range(3):
            if what == "mlp":
                set_weights(2 + i)
            rewind()
            call(many)
            rewind()
            graph.replay()
            for got, exact in zip(state(), want):
                assert torch.equal(got, exact), i
    finally:
        fc.fc_pool_destroy(pool)
