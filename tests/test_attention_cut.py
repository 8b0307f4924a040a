"""How the prompt attention cuts its work (host code, no GPU): the shapes that the GPU tests run reach every kernel and every way of joining."""
import os
import subprocess

import pytest

import paper_2503_17922_amd as W
from paper_2503_17922_amd import build as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F32, BF16, F16 = W.WKV_F32, W.WKV_BF16, W.WKV_F16

# (query heads, KV heads, channels, type, query rows, keys of every sequence)
SHAPES = [
    # blocks of 256 rows, whole
    (32, 8, 128, BF16, [400] * 8, [400] * 8), (32, 8, 128, F16, [401, 390, 5] + [400] * 6, [401, 390, 5] + [400] * 6),
    (32, 8, 64, BF16, [400] * 16, [400] * 16), (32, 8, 64, F16, [399] * 16, [411] * 16),
    # in up to eight parts
    (8, 8, 128, BF16, [4097], [4097]), (32, 8, 128, F16, [250], [9000]), (32, 8, 64, BF16, [300], [6001]), (16, 4, 64, F16, [1000], [7000]),
    # in more
    (8, 4, 128, BF16, [499], [16000]), (8, 4, 128, F16, [512], [15999]), (8, 4, 64, BF16, [500], [16000]), (8, 4, 64, F16, [509], [16001]),
    # blocks of 128 rows: whole, two to a compute unit, in up to eight parts, in more
    (32, 8, 128, BF16, [100], [100]), (28, 4, 64, F16, [333], [333]),
    (32, 8, 128, BF16, [1100], [1100]), (32, 8, 64, F16, [1100], [1100]), (64, 8, 64, F32, [700], [700]), (64, 8, 128, F32, [701], [701]),
    (16, 2, 128, F16, [600, 300], [600, 1500]), (12, 2, 64, BF16, [900], [2000]), (8, 2, 128, F32, [700], [700]), (8, 2, 64, F32, [500], [500]),
    (4, 1, 128, BF16, [1], [9000]), (16, 2, 64, F16, [9, 1], [9000, 77]), (8, 8, 128, F32, [1], [3000]), (8, 2, 64, F32, [3], [5000]),
]


@pytest.fixture(scope="module")
def cuts(tmp_path_factory):
    exe = B.build_host_sanitized(str(tmp_path_factory.mktemp("cut")), [os.path.join(B.CSRC, "wkv_operators.cpp"), os.path.join(ROOT, "tests", "c", "attention_cut.cpp"),
                                                                     os.path.join(ROOT, "tests", "c", "launch_stubs.cpp")], "attention_cut")
    lines = [" ".join(str(x) for x in [len(q), Hq, H, d, t] + [n for pair in zip(q, k) for n in pair]) for Hq, H, d, t, q, k in SHAPES]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0")
    env.pop("LD_PRELOAD", None)
    res = subprocess.run([exe], input="\n".join(lines) + "\n", capture_output=True, text=True, env=env, timeout=300)
    assert res.returncode == 0, res.stdout[-500:] + res.stderr[-2000:]
    return [tuple(int(x) for x in line.split()) for line in res.stdout.splitlines()]


def test_the_shapes_reach_every_kernel(cuts):
    kinds = {}
    for (Hq, H, d, t, q, k), (rows, splits, fold) in zip(SHAPES, cuts):
        kinds.setdefault((t, d, rows), set()).add("whole" if splits == 1 else "few" if splits <= 8 else "many")
        if fold >= 0:
            kinds.setdefault("folded", set()).add((t == F32, d))
            assert rows == 128 and splits == 1
    for d in (64, 128):
        for t in (BF16, F16):
            assert {kind for u in (BF16, F16) for kind in kinds[u, d, 128]} >= {"whole", "few", "many"}
            assert kinds[t, d, 256] == {"whole", "few", "many"}, (t, d, kinds)
        assert kinds[F32, d, 128] >= {"few", "many"} and (F32, d, 256) not in kinds
    assert kinds["folded"] == {(False, 128), (False, 64), (True, 64), (True, 128)}
