"""Options of bench.py that need each other."""
import os
import subprocess
import sys

import pytest
import torch

import workloads as W

BENCH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "bench.py")


@pytest.mark.parametrize("extra", [[], ["--execute"]])
def test_a_cache_without_a_stack_is_refused(extra):
    """(It would run the usual step, as if it had to do with the cache.)"""
    done = subprocess.run([sys.executable, BENCH, "--kv-cache", "4bit"] + extra, capture_output=True, text=True, timeout=100)
    assert done.returncode == 2 and "--stack-report" in done.stderr and done.stdout == ""


@pytest.mark.gpu
def test_the_report_is_of_the_cache_that_is_executed():
    import bench
    import paper_2605_16579_amd as A
    dev = torch.device("cuda:0")
    dense, four = (bench.stack_report(A, W, torch, dev, layers=4, hybrid_layers=2, chunks=2, reps=1, kv_cache=c) for c in ("bf16", "4bit"))
    assert (dense["kv_cache"], four["kv_cache"]) == ("bf16", "4bit")
    # a page of 64 tokens more at most, at 136 bytes of a token and head instead of 512
    w = W.WORKLOADS["wan_layer"]
    assert dense["softmax_stack"]["memory_bytes"] == 4 * 2 * w.L * w.H * 512
    assert four["softmax_stack"]["memory_bytes"] == 4 * -(-2 * w.L // 64) * 64 * w.H * 136
    ex = bench.stack_execute(A, W, torch, dev, layers=4, hybrid_layers=2, chunks=2, kv_cache="4bit")
    for stack in ("hybrid_stack", "softmax_stack"):
        assert 0.5 < ex[stack]["attention_ms"] / four[stack]["attention_ms"] < 2
