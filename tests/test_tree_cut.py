"""Trees of drafted tokens through every kernel there is: which one a shape takes on the CPU (host code), its results on the GPU."""
import math
import os
import random
import subprocess

import pytest

import paper_2503_17922_amd as W
from paper_2503_17922_amd import build as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F32, BF16, F16 = W.WKV_F32, W.WKV_BF16, W.WKV_F16

# (batch, query heads, KV heads, channels, nodes, capacity); waves along the rows, how the ranges are joined, whether the caches are read past the memory-side cache.
# Blocks of 256 rows one and two to a pair, full and not.  (Of several ranges they are never cut into.)
HALF = [
    ((3, 16, 16, 128, 33, 100), (2, "whole", 0)), ((3, 64, 8, 128, 1, 400), (2, "few", 0)), ((1, 28, 4, 128, 9, 5000), (2, "many", 0)),
    ((40, 64, 8, 128, 7, 2000), (2, "whole", 1)), ((16, 32, 8, 128, 5, 5000), (2, "few", 1)), ((1, 32, 8, 128, 16, 140000), (2, "many", 1)),
    ((8, 8, 2, 128, 33, 400), (4, "whole", 0)), ((3, 28, 4, 128, 64, 1500), (4, "few", 0)), ((3, 8, 2, 128, 64, 5000), (4, "many", 0)),
    ((40, 28, 4, 128, 33, 5000), (4, "whole", 1)), ((8, 28, 4, 128, 16, 20000), (4, "few", 1)), ((1, 32, 8, 128, 60, 140000), (4, "many", 1)),
    ((35, 32, 8, 128, 64, 100), (8, "whole", 0)), ((33, 64, 8, 128, 61, 150), (8, "whole", 0)), ((70, 28, 4, 128, 33, 2000), (8, "whole", 1)),
    ((8, 8, 2, 64, 16, 400), (2, "whole", 0)), ((3, 32, 8, 64, 16, 1500), (2, "few", 0)), ((3, 12, 2, 64, 7, 5000), (2, "many", 0)),
    ((40, 64, 8, 64, 5, 4000), (2, "whole", 1)), ((40, 28, 4, 64, 7, 20000), (2, "few", 1)), ((3, 32, 8, 64, 16, 70000), (2, "many", 1)),
    ((8, 28, 4, 64, 33, 100), (4, "whole", 0)), ((8, 28, 4, 64, 33, 1500), (4, "few", 0)), ((1, 64, 8, 64, 33, 5000), (4, "many", 0)),
    ((70, 28, 4, 64, 16, 5000), (4, "whole", 1)), ((8, 32, 8, 64, 33, 20000), (4, "few", 1)), ((1, 32, 8, 64, 50, 140000), (4, "many", 1)),
    ((40, 32, 8, 64, 64, 130), (8, "whole", 0)), ((35, 64, 8, 64, 61, 100), (8, "whole", 0)), ((70, 28, 4, 64, 33, 5000), (8, "whole", 1)),
]
FULL = [
    ((3, 16, 16, 128, 33, 100), (2, "whole", 0)), ((1, 8, 1, 128, 1, 400), (2, "few", 0)), ((1, 16, 16, 128, 16, 1500), (2, "many", 0)),
    ((40, 64, 8, 128, 7, 1500), (2, "whole", 1)), ((8, 32, 8, 128, 7, 5000), (2, "few", 1)), ((1, 32, 8, 128, 9, 70000), (2, "many", 1)),
    ((16, 32, 8, 128, 64, 100), (4, "whole", 0)), ((1, 32, 8, 128, 33, 400), (4, "few", 0)), ((1, 8, 1, 128, 33, 9000), (4, "many", 0)),
    ((70, 32, 8, 128, 33, 1500), (4, "whole", 1)), ((8, 28, 4, 128, 64, 9000), (4, "few", 1)), ((1, 64, 8, 128, 16, 70000), (4, "many", 1)),
    ((3, 16, 16, 64, 1, 100), (2, "whole", 0)), ((3, 16, 16, 64, 1, 400), (2, "few", 0)), ((3, 64, 8, 64, 1, 1500), (2, "many", 0)),
    ((70, 32, 8, 64, 7, 1500), (2, "whole", 1)), ((16, 16, 16, 64, 64, 5000), (2, "few", 1)), ((1, 32, 8, 64, 16, 140000), (2, "many", 1)),
    ((16, 64, 8, 64, 16, 100), (4, "whole", 0)), ((1, 64, 8, 64, 64, 400), (4, "few", 0)), ((16, 8, 1, 64, 16, 1500), (4, "many", 0)),
    ((70, 28, 4, 64, 33, 5000), (4, "whole", 1)), ((70, 8, 1, 64, 33, 9000), (4, "few", 1)), ((1, 32, 8, 64, 33, 140000), (4, "many", 1)),
]
SHAPES = [(t, *shape, kind) for t in (BF16, F16) for shape, kind in HALF] + [(F32, *shape, kind) for shape, kind in FULL]


def test_the_shapes_reach_every_kernel(tmp_path):
    exe = B.build_host_sanitized(str(tmp_path), [os.path.join(B.CSRC, f) for f in ("wkv_operators.cpp", "wkv_generation.cpp")] +
                                 [os.path.join(ROOT, "tests", "c", f) for f in ("tree_cut.cpp", "launch_stubs.cpp")], "tree_cut")
    lines = [" ".join(str(x) for x in (b, Hq, H, d, t, T, cap)) for t, b, Hq, H, d, T, cap, _ in SHAPES]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0")
    env.pop("LD_PRELOAD", None)
    res = subprocess.run([exe], input="\n".join(lines) + "\n", capture_output=True, text=True, env=env, timeout=300)
    assert res.returncode == 0, res.stdout[-500:] + res.stderr[-2000:]
    cuts = [tuple(int(x) for x in line.split()) for line in res.stdout.splitlines()]
    assert len(cuts) == len(SHAPES)
    blocks = {}
    for (t, b, Hq, H, d, T, cap, kind), (row_waves, key_waves, n_blocks, splits, streams) in zip(SHAPES, cuts):
        assert (row_waves, "whole" if splits == 1 else "few" if splits <= 8 else "many", streams) == kind, (t, b, Hq, H, d, T, cap)
        blocks.setdefault((t, d, row_waves), set()).add(n_blocks)
    for t in (BF16, F16, F32):
        for d in (64, 128):
            kinds = {s[-1] for s in SHAPES if s[0] == t and s[4] == d}
            assert kinds == {(r, join, s) for r in (2, 4) for join in ("whole", "few", "many") for s in (0, 1)} | ({(8, "whole", s) for s in (0, 1)} if t != F32 else set())
            assert len(blocks[t, d, 4]) > 1
            assert t == F32 or blocks[t, d, 8] == {1, 2}


def some_counts(B_, cap, T, seed):
    """Lengths of all sizes; one cache without room for the tree where there are several."""
    r = random.Random(seed)
    most = min(cap - T, 3000)
    out = [r.choice([0, 1, 63, 64, 65, 127, 128, most, r.randrange(most + 1), r.randrange(most + 1)]) for _ in range(B_)]
    out = [min(n, cap - T) for n in out]
    out[0] = cap - T if cap <= 20000 else 9000
    if B_ > 2:
        out[1] = cap - T + 1
    return out


@pytest.mark.gpu
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(str(x) for x in s[:7]) + "-" + "-".join(str(x) for x in s[7]))
def test_results(device, shape):
    import torch

    from tests.test_gpu_tree import families, some_tree
    dtype, B_, Hq, H, d, T, cap, _ = shape
    t = {F32: torch.float32, BF16: torch.bfloat16, F16: torch.float16}[dtype]
    half, G, scale = torch.finfo(t).eps / 2, Hq // H, d ** -0.5
    g = torch.Generator(device=device).manual_seed(60)
    r = random.Random(61)
    counts = some_counts(B_, cap, T, 62)
    parents = [some_tree(T, b) for b in range(B_)]
    for b in range(0, B_, 3):                                  # padding: behind the tree, and in it
        parents[b] = parents[b][:max(T - 2, 1)] + [-2] * (T - max(T - 2, 1))
        if T > 5:
            parents[b][r.randrange(1, T - 2)] = 1000
    q, kn, vn = ((torch.randn((B_, n, T, d), device=device, generator=g) * s).to(t) for n, s in ((Hq, 1.5), (H, 1.0), (H, 1.0)))
    fam = [families(p) for p in parents]
    for b in range(B_):                                        # what padding holds shows nowhere
        gone = [i for i in range(T) if fam[b][i] is None]
        q[b, :, gone], kn[b, :, gone], vn[b, :, gone] = math.nan, math.inf, math.nan
    # a node whose value is not finite: one sequence, one head
    odd = (B_ - 1, H - 1, 0)
    if fam[odd[0]][0] is not None:
        vn[odd[0], odd[1], 0, 5] = math.inf
    kc, vc = (torch.full((B_, H, cap, d), math.nan, dtype=t, device=device) for _ in range(2))
    for b, n in enumerate(counts):
        for c in (kc, vc):
            c[b, :, :n] = torch.randn((H, min(n, cap), d), device=device, generator=g).to(t)
    n_valid = torch.tensor(counts, dtype=torch.int32, device=device)[:, None].repeat(1, H)
    out = torch.full((B_, Hq, T, d), 7.0, dtype=t, device=device)
    sh = W.TreeShape(batch=B_, n_q_heads=Hq, n_kv_heads=H, head_dim=d, dtype=dtype, n_nodes=T, capacity=cap)
    ws = torch.full((W.wkv_tree_workspace_bytes(sh),), 0xff, dtype=torch.uint8, device=device)
    W.wkv_decode_tree(sh, q, kn, vn, torch.tensor(parents, dtype=torch.int32, device=device), kc, vc, n_valid, out, ws)
    torch.cuda.synchronize()
    # tolerances as in test_gpu_tree_rounding.py
    parts = {F32: 0.0, BF16: 2.0 ** -15, F16: 2.0 ** -20}[dtype]
    pairs = [(b, h) for b in range(B_) for h in range(H)]
    pairs = pairs if len(pairs) <= 24 else [pairs[0], pairs[H], pairs[-1]] + r.sample(pairs, 20)
    for b, h in pairs:
        n = counts[b]
        nodes = [i for i in range(T) if fam[b][i] is not None]
        gone = [i for i in range(T) if fam[b][i] is None]
        got = out[b, h * G:(h + 1) * G]
        assert (got[:, gone] == 7.0).all()
        if n + T > cap:
            assert torch.isnan(got[:, nodes]).all() and torch.isnan(kc[b, h, n:]).all() and torch.isnan(vc[b, h, n:]).all()
            continue
        assert torch.equal(kc[b, h, [n + i for i in nodes]], kn[b, h, nodes]) and torch.equal(vc[b, h, [n + i for i in nodes]], vn[b, h, nodes])
        for c in (kc, vc):
            assert torch.isnan(c[b, h, [n + i for i in gone] + list(range(n + T, min(cap, n + T + 50)))]).all()
        hidden = torch.ones((len(nodes), n + T), dtype=torch.bool)
        hidden[:, :n] = False
        for row, i in enumerate(nodes):
            hidden[row, [n + j for j in fam[b][i]]] = False
        hidden = hidden.to(device)
        k, v = (torch.cat([c[b, h, :n], x[b, h]]).double() for c, x in ((kc, kn), (vc, vn)))
        wrong = ~torch.isfinite(v).all(-1)
        wrong[[n + i for i in gone]] = False
        sees = (~hidden & wrong).any(-1)                       # these rows are NaN, and no others
        assert torch.isnan(got[:, nodes][:, sees]).all()
        k, v = k.nan_to_num(posinf=0.0), v.nan_to_num(posinf=0.0)
        x = q[b, h * G:(h + 1) * G][:, nodes].double()
        p = torch.softmax((x @ k.t() * scale).masked_fill(hidden, -math.inf), -1)
        want, size = p @ v, p @ v.abs()
        delta = (d + 4) * 2.0 ** -24 * scale * x.norm(dim=-1) * k.norm(dim=-1).max()
        loose = 2 * delta + (2 * (n + T) + 128) * 2.0 ** -24
        tol = want.abs() * half + size * (parts + loose[..., None]) * (1 + half) + (n + T) * 2.0 ** -37 * v.abs().amax() + (2.0 ** -25 if dtype == F16 else 1e-38)
        err = (got[:, nodes].double() - want).abs()[:, ~sees]
        assert (err <= tol[:, ~sees]).all(), f"({b}, {h}): worst {float((err / tol[:, ~sees]).max())} of the tolerance"
    del kc, vc
