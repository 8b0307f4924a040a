"""wkv_decode_tree in 16 bits rounds nothing but its output: against 64 bits, with what the types' own rounding allows and no more."""
import math

import pytest
import torch

import paper_2503_17922_amd as W
from tests.test_gpu_tree import TYPES, Tree, families, some_tree

pytestmark = pytest.mark.gpu

# (counts, query heads, KV heads, channels, nodes): blocks of 64, 128 and 256 rows; one range, a few, many
SHAPES = [([300, 77], 8, 2, 128, 16), ([4128], 32, 8, 128, 16), ([333, 0], 28, 4, 64, 20), ([900, 2000], 28, 4, 128, 64), ([200] * 40, 32, 8, 128, 64),
          ([150] * 70, 16, 8, 64, 1)]


@pytest.mark.parametrize("dtype", [W.WKV_BF16, W.WKV_F16])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"{len(s[0])}x{s[0][0]}-{s[1]}-{s[2]}-{s[3]}-{s[4]}")
def test_only_the_output_is_rounded(device, dtype, shape):
    counts, Hq, H, d, T = shape
    s = Tree(device, counts, [some_tree(T, b) for b in range(len(counts))], Hq, H, d, dtype, max(counts) + T, seed=31)
    s.step()
    torch.cuda.synchronize()
    G, t = Hq // H, TYPES[dtype]
    half = torch.finfo(t).eps / 2
    # A probability reaches the product as two numbers of the type, what the first leaves over in the second: 8 + 8 bits (2^-15 of it are left when both are cut off),
    # 11 + 11 (2^-20; in fp16 numbers below 2^-14 have fewer bits, 2^-24 of a reference that is 2^13 and more: 2^-37 of the row's sum).
    parts = 2.0 ** -15 if dtype == W.WKV_BF16 else 2.0 ** -20
    off = total = 0.0
    for b, n in enumerate(counts):
        fam = families(s.parents[b])
        hidden = torch.ones((T, n + T), dtype=torch.bool, device=device)
        hidden[:, :n] = False
        for i, f in enumerate(fam):
            hidden[i, [n + j for j in f]] = False
        for h in range(H):
            k, v = (torch.cat([c[b, h, :n], x[b, h]]).double() for c, x in ((s.kc[0], s.kn), (s.vc[0], s.vn)))
            q = s.q[b, h * G:(h + 1) * G].double()
            p = torch.softmax((q @ k.t() * d ** -0.5).masked_fill(hidden, -math.inf), -1)
            want, size = p @ v, p @ v.abs()
            # logits, sums and joins as in test_gpu_tree.py
            delta = (d + 4) * 2.0 ** -24 * d ** -0.5 * q.norm(dim=-1) * k.norm(dim=-1).max()
            loose = 2 * delta + (2 * (n + T) + 128) * 2.0 ** -24
            exact = size * (parts + loose[..., None])
            tol = want.abs() * half + exact * (1 + half) + (n + T) * 2.0 ** -37 * v.abs().amax() + (2.0 ** -25 if t == torch.float16 else 1e-38)
            err = (s.out[b, h * G:(h + 1) * G].double() - want).abs()
            assert (err <= tol).all(), f"({b}, {h}): worst {float((err / tol).max())} of the tolerance"
            off += float((err ** 2).sum())
            total += float(((want.to(t).double() - want) ** 2).sum())
    # and the root of the mean square is that of numbers rounded to the type: an error of 2^-15 at random beside one of 2^-8 adds 2^-14 of its square, and an
    # average over 10^4 numbers and more leaves 1 %
    assert off <= total * 1.02, math.sqrt(off / total)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("Hq,H,d,T,counts", [(8, 2, 128, 16, [300, 77]), (28, 4, 128, 40, [1000, 400]), (8, 2, 64, 40, [1500]), (32, 8, 128, 64, [120] * 33)])
def test_a_row_does_not_depend_on_the_rows_beside_it(device, dtype, Hq, H, d, T, counts):
    """Queries of other nodes, and what padding holds, change no bit of a node's output."""
    parents = [some_tree(T, b) for b in range(len(counts))]
    for p in parents:
        p[T - 1] = -2                                          # one that does not exist
    s = Tree(device, counts, parents, Hq, H, d, dtype, max(counts) + T, seed=32)
    kept = list(range(0, T - 1, 3))
    others = [i for i in range(T) if i not in kept]
    s.step()
    torch.cuda.synchronize()
    first = s.out[:, :, kept].clone()
    cache = [s.kc[0].clone(), s.vc[0].clone()]
    for factor in (0.0, 6.0, -6.0, math.nan):
        s.kc[0].copy_(cache[0])
        s.vc[0].copy_(cache[1])
        changed = s.q[:, :, others] * factor if factor == factor else torch.full_like(s.q[:, :, others], math.nan)
        was = s.q[:, :, others].clone()
        s.q[:, :, others] = changed
        s.step()
        torch.cuda.synchronize()
        s.q[:, :, others] = was
        assert torch.equal(s.out[:, :, kept], first), factor


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("T,counts", [(16, [200, 3000]), (64, [700, 90])])
def test_the_largest_logits(device, dtype, T, counts):
    """Up to 10^7: a row is the value of its largest logit, where the others are a step of fp32's logits and more below."""
    d = 128
    s = Tree(device, counts, [some_tree(T, b) for b in range(2)], 8, 2, d, dtype, max(counts) + T, seed=33, spread=1.0, scale=1.0)
    # queries of one channel, keys of -1 .. 1 in it: logits of 9.8e6 at most
    big = 9.8e6 if dtype != W.WKV_F16 else 6.0e4
    s.q.zero_()
    s.q[..., 3] = big
    for c in (s.kc[0], s.kn):
        c[..., 3] = -c[..., 3].abs().clamp(0.25, 0.9)
    scale = big / 9.8e6 if dtype != W.WKV_F16 else 9.8e6 / 6.0e4
    top = [37, 60]                                             # a row of the cache
    for b in range(2):
        s.kc[0][b, :, top[b], 3] = 1.0
    s.shape.c.scale = scale
    s.step()
    torch.cuda.synchronize()
    for b in range(2):
        want = s.vc[0][b, :, top[b]].repeat_interleave(4, 0)[:, None].expand(-1, T, -1)
        # p v / p: the products with the value, the reciprocal and its product, and two rescalings of either side where ranges are joined: eight steps of 2^-24.  (A value of a 16-bit
        # type is itself again when that is rounded to the type.)
        if dtype == W.WKV_F32:
            assert ((s.out[b].double() - want.double()).abs() <= want.double().abs() * 2.0 ** -21).all(), b
        else:
            assert torch.equal(s.out[b], want), b
