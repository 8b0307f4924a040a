"""Blocks of 128 rows of the prompt attention, for each 16-bit type and head size by itself (their kernels are compiled apart): whole, joined by one group of threads
and by eight.  The cuts on the CPU, the results on the GPU."""
import os
import subprocess

import pytest

import paper_2503_17922_amd as W
from paper_2503_17922_amd import build as B
from tests.test_attention_cut import ROOT

# (query heads, KV heads, query rows, keys): the kind of cut
CUTS = {"whole": [(32, 8, [100], [100]), (8, 2, [333], [333])],
        "few": [(12, 2, [900], [2000]), (16, 2, [600, 300], [600, 1500])],
        "many": [(4, 1, [1], [9000]), (16, 2, [9, 1], [9000, 77])]}
SHAPES = [(kind, Hq, H, d, t, q, k) for t in (W.WKV_BF16, W.WKV_F16) for d in (64, 128) for kind, cuts in CUTS.items() for Hq, H, q, k in cuts]


def test_cuts(tmp_path):
    exe = B.build_host_sanitized(str(tmp_path), [os.path.join(B.CSRC, "wkv_operators.cpp"), os.path.join(ROOT, "tests", "c", "attention_cut.cpp"),
                                                 os.path.join(ROOT, "tests", "c", "launch_stubs.cpp")], "attention_cut")
    lines = [" ".join(str(x) for x in [len(q), Hq, H, d, t] + [n for pair in zip(q, k) for n in pair]) for _, Hq, H, d, t, q, k in SHAPES]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0")
    env.pop("LD_PRELOAD", None)
    res = subprocess.run([exe], input="\n".join(lines) + "\n", capture_output=True, text=True, env=env, timeout=300)
    assert res.returncode == 0, res.stdout[-500:] + res.stderr[-2000:]
    cuts = [[int(x) for x in line.split()] for line in res.stdout.splitlines()]
    assert len(cuts) == len(SHAPES)
    for (kind, *_), (rows, splits, _) in zip(SHAPES, cuts):
        assert (rows, "whole" if splits == 1 else "few" if splits <= 8 else "many") == (128, kind)


@pytest.mark.gpu
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(str(x) for x in s[:5]) + f"-{s[5][0]}")
def test_results(device, shape):
    from tests.test_gpu_prefill_attention import run
    _, Hq, H, d, dtype, q_len, k_len = shape
    run(device, q_len, k_len, Hq, H, d, dtype, lse_rows=7, seed=len(q_len))
