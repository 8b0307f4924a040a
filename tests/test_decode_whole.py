"""Where the weighted decode step gives a whole cache to one workgroup and where ranges of it to several (host code, no GPU): the rule's borders, and
that the shapes of the GPU tests are on the side that these tests are about."""
import os
import subprocess

import pytest

import paper_2503_17922_amd as W
from paper_2503_17922_amd import build as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F32, BF16, F16 = W.WKV_F32, W.WKV_BF16, W.WKV_F16

# (batch, query heads, KV heads, channels, type, capacity): what tests/test_gpu_decode_whole.py and the tests of a workgroup a cache in tests/test_gpu_decode_weighted.py run
WHOLE = [(b, hq, h, d, t, cap) for t in (BF16, F16) for b, hq, h, d, cap in [
    (64, 16, 4, 128, 300), (7, 32, 32, 128, 700), (52, 64, 8, 64, 200), (56, 24, 8, 128, 130), (60, 20, 4, 64, 4032), (56, 16, 4, 128, 5056), (128, 14, 2, 64, 17),
    (7, 64, 32, 64, 10112), (56, 16, 4, 128, 128), (130, 16, 4, 128, 700), (65, 8, 8, 128, 500), (29, 16, 8, 128, 10112), (28, 8, 8, 128, 10112), (28, 8, 8, 64, 20224), (8, 32, 32, 128, 300)]]
RANGES = [(b, hq, h, d, t, cap) for t in (BF16, F16) for b, hq, h, d, cap in [
    (28, 8, 8, 128, 10113), (28, 8, 8, 128, 20224), (28, 8, 8, 64, 20225), (28, 16, 8, 128, 10113), (52, 32, 8, 128, 5057), (28, 40, 8, 128, 300), (33, 32, 8, 128, 1000),
    (51, 32, 8, 128, 1000), (27, 32, 8, 128, 1000), (1, 4, 1, 128, 257)]] + [(64, 32, 8, 128, F32, 300), (1, 4, 1, 64, F32, 20)]
SHORT = [(1, 4, 1, 128, BF16, 256), (1, 8, 1, 64, F16, 1), (40, 32, 8, 128, F16, 256)]


def test_who_takes_a_cache(tmp_path):
    exe = B.build_host_sanitized(str(tmp_path), [os.path.join(B.CSRC, "wkv_operators.cpp"), os.path.join(ROOT, "tests", "c", "decode_whole.cpp"),
                                                 os.path.join(ROOT, "tests", "c", "launch_stubs.cpp")], "decode_whole")
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0")
    env.pop("LD_PRELOAD", None)
    shapes = WHOLE + SHORT + RANGES
    res = subprocess.run([exe], input="".join(" ".join(str(x) for x in s) + "\n" for s in shapes), capture_output=True, text=True, env=env, timeout=300)
    assert res.returncode == 0, res.stdout[-500:] + res.stderr[-2000:]
    got = [line == "1" for line in res.stdout.split()]
    assert got == [True] * (len(WHOLE) + len(SHORT)) + [False] * len(RANGES), [s for s, g in zip(shapes, got) if g == (s in RANGES)]
