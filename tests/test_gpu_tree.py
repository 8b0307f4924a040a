"""wkv_decode_tree against softmax(q K^T scale) V in 64 bits over the cache and a node's ancestors, and wkv_tree_accept row by row."""
import math
import random

import pytest
import torch

import paper_2503_17922_amd as W

pytestmark = pytest.mark.gpu

TYPES = {W.WKV_F32: torch.float32, W.WKV_BF16: torch.bfloat16, W.WKV_F16: torch.float16}


def chain(T):
    return [t - 1 for t in range(T)]


def some_tree(T, seed):
    r = random.Random(seed)
    return [r.randrange(-1, t) if r.random() < 0.6 else t - 1 for t in range(T)]


def families(parent):
    """A node's row of numbers: itself and those it hangs below; None: it does not exist."""
    out = []
    for t, p in enumerate(parent):
        if p == -1:
            out.append([t])
        elif 0 <= p < t and out[p] is not None:
            out.append(out[p] + [t])
        else:
            out.append(None)
    return out


class Tree:
    def __init__(self, device, counts, parents, Hq, H, d, dtype, cap, seed=1, layout="projection", spread=1.5, scale=0.0, flags=0, layers=1, values=None):
        g = torch.Generator(device=device).manual_seed(seed)
        B, T, t = len(counts), len(parents[0]), TYPES[dtype]
        randn = lambda *s: torch.randn(s, device=device, generator=g)
        self.n = torch.tensor(counts, dtype=torch.int32, device=device)
        if self.n.dim() == 1:
            self.n = self.n[:, None].repeat(1, H)
        c_strides = None
        if layout == "projection":                             # q, k, v of a token in one row; rows of the cache by head
            w = Hq + 2 * H
            rows = torch.cat([randn(B, T, Hq, d) * spread, randn(B, T, 2 * H, d)], 2).to(t)
            self.q, self.kn, self.vn = (x.transpose(1, 2) for x in (rows[:, :, :Hq], rows[:, :, Hq:Hq + H], rows[:, :, Hq + H:]))
            q_strides = new_strides = (T * w * d, d, w * d)
            self.out = torch.full((B, T, Hq, d), 7.0, dtype=t, device=device).transpose(1, 2)
            out_strides = (T * Hq * d, d, Hq * d)
            self.kc, self.vc = ([randn(B, H, cap, d).to(t) for _ in range(layers)] for _ in range(2))
        else:                                                  # by head; the cache by token, rows d + 16 elements apart
            self.q, self.kn, self.vn = (randn(B, Hq, T, d) * spread).to(t), randn(B, H, T, d).to(t), randn(B, H, T, d).to(t)
            q_strides = new_strides = None
            self.out = torch.full((B, Hq, T, d), 7.0, dtype=t, device=device)
            out_strides = (Hq * T * d, T * d, d)
            c_strides = (cap * H * (d + 16), d + 16, H * (d + 16))
            self.kc, self.vc = ([randn(B, cap, H, d + 16).to(t).transpose(1, 2)[..., :d] for _ in range(layers)] for _ in range(2))
        for c in self.kc + self.vc:                            # rows from the count on may hold anything
            for b in range(B):
                for h in range(H):
                    c[b, h, min(max(int(self.n[b, h]), 0), cap):] = math.nan
        if values:
            values(self)
        self.parents = parents
        self.parent = torch.tensor(parents, dtype=torch.int32, device=device)
        self.shape = W.TreeShape(batch=B, n_q_heads=Hq, n_kv_heads=H, head_dim=d, dtype=dtype, n_nodes=T, capacity=cap, scale=scale, cache_strides=c_strides,
                                 q_strides=q_strides, new_strides=new_strides, out_strides=out_strides, flags=flags)
        self.ws = torch.full((W.wkv_tree_workspace_bytes(self.shape),), 0xff, dtype=torch.uint8, device=device)
        self.cap, self.dtype, self.scale = cap, dtype, scale or d ** -0.5

    def step(self, layer=0):
        W.wkv_decode_tree(self.shape, self.q, self.kn, self.vn, self.parent, self.kc[layer], self.vc[layer], self.n, self.out, self.ws)

    def check(self, layer=0):
        before = [self.kc[layer].clone(), self.vc[layer].clone(), self.n.clone(), self.out.clone()]
        self.step(layer)
        torch.cuda.synchronize()
        self.compare(before, layer)

    def compare(self, before, layer=0):
        kc, vc, counts, old = before
        B, Hq, T, d = self.q.shape
        H = kc.shape[1]
        G = Hq // H
        t = TYPES[self.dtype]
        half = torch.finfo(t).eps / 2
        assert torch.equal(self.n, counts)
        for b in range(B):
            fam = families(self.parents[b])
            nodes = [i for i in range(T) if fam[i] is not None]
            gone = [i for i in range(T) if fam[i] is None]
            for h in range(H):
                n = int(counts[b, h])
                got = self.out[b, h * G:(h + 1) * G]
                assert torch.equal(got[:, gone], old[b, h * G:(h + 1) * G][:, gone]), "rows of nodes that do not exist"
                if n < 0 or n + T > self.cap:
                    assert torch.isnan(got[:, nodes]).all(), (b, h)
                    continue
                for i in nodes:
                    kc[b, h, n + i], vc[b, h, n + i] = self.kn[b, h, i], self.vn[b, h, i]
                if not nodes:
                    continue
                k, v = kc[b, h, :n + T].double().nan_to_num(), vc[b, h, :n + T].double().nan_to_num()
                hidden = torch.ones((len(nodes), n + T), dtype=torch.bool)
                hidden[:, :n] = False
                for r, i in enumerate(nodes):
                    hidden[r, [n + j for j in fam[i]]] = False
                hidden = hidden.to(k.device)
                q = self.q[b, h * G:(h + 1) * G][:, nodes].double()
                s = (q @ k.t() * self.scale).masked_fill(hidden, -math.inf)
                p = torch.softmax(s, -1)
                want, size = p @ v, p @ v.abs()
                # as for the prompt's attention: a logit is off by (d + 4) 2^-24 scale |q| |k|, a probability by twice that, sums of m probabilities and
                # products by m 2^-24 each, the joins of up to 64 ranges and the exponents by 2^-17 together; 16-bit types round every probability by half a
                # step, and every type the output once
                m = n + T
                delta = (d + 4) * 2.0 ** -24 * self.scale * q.norm(dim=-1) * k.norm(dim=-1).max()
                loose = 2 * delta + (2 * m + 128) * 2.0 ** -24
                tol = want.abs() * half + size * ((half if self.dtype != W.WKV_F32 else 0.0) + loose[..., None]) * (1 + half) + (2.0 ** -24 if self.dtype == W.WKV_F16 else 1e-38)
                err = (got[:, nodes].double() - want).abs()
                assert (err <= tol).all(), f"({b}, {h}): worst {float((err / tol).max())} of the tolerance"
        for x, y in ((self.kc[layer], kc), (self.vc[layer], vc)):
            assert torch.equal(torch.isnan(x), torch.isnan(y)) and torch.equal(x.nan_to_num(), y.nan_to_num()), "the caches"


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hq,H", [(2, 2), (8, 2), (7, 1), (16, 2)])
@pytest.mark.parametrize("T", [1, 5, 16, 33, 64])
def test_types_heads_and_nodes(device, dtype, d, Hq, H, T):
    Tree(device, [0, 1, 200, 333], [some_tree(T, 10 * T + b) for b in range(4)], Hq, H, d, dtype, 400, seed=T).check()


@pytest.mark.parametrize("T", [1, 9, 40, 64])
@pytest.mark.parametrize("n", [0, 1, 31, 32, 33, 63, 64, 65, 127, 128, 129, 191, 1000, 4128])
def test_lengths(device, T, n):
    Tree(device, [n], [some_tree(T, n)], 8, 2, 128, W.WKV_BF16, n + T, seed=n + 1).check()


@pytest.mark.parametrize("shape", ["chain", "star", "comb", "pairs"])
@pytest.mark.parametrize("T", [2, 31, 64])
def test_shapes_of_trees(device, shape, T):
    parent = {"chain": chain(T), "star": [-1] * T, "comb": [t - 1 if t % 2 else max(t - 2, -1) for t in range(T)], "pairs": [(t - 1) // 2 if t else -1 for t in range(T)]}[shape]
    for dtype in TYPES:
        Tree(device, [70, 3], [parent, parent], 4, 1, 64, dtype, 200, seed=T).check()


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("T", [7, 64])
def test_nodes_that_do_not_exist(device, dtype, T):
    # padding behind the tree, parents that come later, hang below nothing or below themselves, whole trees of none
    a = some_tree(T, 3); a[T // 2:] = [-2] * (T - T // 2)
    b = some_tree(T, 4); b[2] = 2; b[3] = 2; b[4] = 5
    c = [-2] * T
    e = some_tree(T, 5); e[0] = 1000; e[1] = -2 ** 31
    Tree(device, [100, 0, 90, 257], [a, b, c, e], 8, 2, 128, dtype, 400, seed=T).check()


@pytest.mark.parametrize("dtype,d,Hq,H,T", [(W.WKV_BF16, 128, 32, 8, 16), (W.WKV_F16, 128, 28, 4, 64), (W.WKV_F32, 64, 12, 2, 20), (W.WKV_BF16, 64, 32, 32, 8),
                                            (W.WKV_F32, 128, 8, 1, 64)])
@pytest.mark.parametrize("layout", ["projection", "heads"])
def test_batches_of_mixed_lengths(device, dtype, d, Hq, H, T, layout):
    counts = [0, 700, 3, 2000, 64, 1999, 2048 - T, 2049 - T, 2048, -1]          # three have no room for the tree
    Tree(device, counts, [some_tree(T, b) for b in range(len(counts))], Hq, H, d, dtype, 2048, seed=7, layout=layout).check()


def test_counts_of_their_own_for_each_head(device):
    Tree(device, [[5, 0, 290], [301, 77, -7], [128, 32, 285]], [some_tree(16, b) for b in range(3)], 12, 3, 128, W.WKV_BF16, 301, seed=8).check()


@pytest.mark.parametrize("spread,scale", [(40.0, 0.0), (1.0, 3.0), (0.0, 0.0)])
@pytest.mark.parametrize("dtype", list(TYPES))
def test_logits_of_all_sizes(device, dtype, spread, scale):
    Tree(device, [500, 77], [some_tree(24, b) for b in range(2)], 8, 2, 128, dtype, 600, seed=10, spread=spread, scale=scale).check()


def test_one_node_that_outweighs_a_row(device):
    # in fp16 a key of value zero far above the others: what is left of them still counts
    def values(s):
        s.kn[:, :, 0] = s.q[:, 0::8, 1].to(s.kn.dtype) * 2
        s.vn[:, :, 0] = 0.0
    Tree(device, [1000], [[-1, 0, 0, 1]], 8, 1, 128, W.WKV_F16, 1100, seed=11, spread=1.0, values=values).check()


def test_a_chain_is_a_prompt(device):
    # the same rows through wkv_prefill_attention
    T, n, Hq, H, d = 40, 500, 8, 2, 128
    s = Tree(device, [n], [chain(T)], Hq, H, d, W.WKV_F32, n + T, seed=12, layout="heads")
    s.check()
    k, v = s.kc[0].contiguous(), s.vc[0].contiguous()
    a = W.AttentionShape(q_len=[T], k_len=[n + T], n_q_heads=Hq, n_kv_heads=H, head_dim=d, dtype=W.WKV_F32)
    out = torch.zeros((1, Hq, T, d), device=device)
    W.wkv_prefill_attention(a, s.q, k, v, out, None, torch.empty(W.wkv_attention_workspace_bytes(a), dtype=torch.uint8, device=device))
    assert torch.allclose(out, s.out, rtol=1e-4, atol=1e-5)


def test_one_node_is_a_decode_step(device):
    s = Tree(device, [300, 77], [[-1], [-1]], 8, 2, 128, W.WKV_F32, 301, seed=13)
    kc, vc, n = s.kc[0].clone(), s.vc[0].clone(), s.n.clone()
    s.check()
    sh = W.DecodeShape(batch=2, n_q_heads=8, n_kv_heads=2, head_dim=128, dtype=W.WKV_F32, capacity=301)
    out = torch.zeros((2, 8, 128), device=device)
    W.wkv_decode_step(sh, s.q[:, :, 0].contiguous(), s.kn[:, :, 0].contiguous(), s.vn[:, :, 0].contiguous(), kc, vc, n, out,
                      torch.empty(W.wkv_decode_workspace_bytes(sh), dtype=torch.uint8, device=device))
    assert torch.allclose(out, s.out[:, :, 0], rtol=1e-4, atol=1e-5)
    assert torch.equal(kc.nan_to_num(), s.kc[0].nan_to_num())


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("T", [4, 40, 64])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_values_that_are_not_finite_stay_with_the_nodes_that_see_them(device, dtype, T, value):
    parent = some_tree(T, 14)
    for n in (0, 100, 1500):
        s = Tree(device, [n, n], [parent, parent], 4, 1, 128, dtype, 1600, seed=14)
        at = [1, T - 1]
        for i in at:
            s.vn[0, 0, i, 3 + i] = value
        s.step()
        bad = ~torch.isfinite(s.out)
        assert not bad[1].any()
        for i, f in enumerate(families(parent)):
            assert bad[0, :, i].all() if set(f) & set(at) else not bad[0, :, i].any(), i
        # a key that is not finite is another matter: the logit of the rows that see it
        s = Tree(device, [n, n], [parent, parent], 4, 1, 128, dtype, 1600, seed=15)
        s.kn[0, 0, 1, 5] = math.nan
        s.step()
        bad = ~torch.isfinite(s.out)
        assert not bad[1].any()
        for i, f in enumerate(families(parent)):
            assert bad[0, :, i].all() if 1 in f else not bad[0, :, i].any(), i


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("T", [3, 33, 64])
def test_what_padding_holds_shows_nowhere(device, dtype, T):
    parent = some_tree(T, 6)
    for i in (1, T - 1):
        parent[i] = -2

    def values(s):
        for i, f in enumerate(families(parent)):
            if f is None:
                s.q[:, :, i] = math.nan
                s.kn[:, :, i] = math.inf
                s.vn[:, :, i] = math.nan
    Tree(device, [100, 0], [parent, parent], 8, 2, 64, dtype, 200, seed=T, values=values).check()


def test_captured_and_replayed(device):
    s = Tree(device, [100, 3000, 0], [some_tree(16, b) for b in range(3)], 8, 2, 128, W.WKV_BF16, 3100, seed=15)
    path = torch.tensor([[0, 1] + [-1] * 14] * 3, dtype=torch.int32, device=device)
    accept = torch.tensor([0, 1, 0], dtype=torch.int32, device=device)

    def both():
        s.step()
        W.wkv_tree_accept(s.shape, s.kc, s.vc, path, accept, s.n)

    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for turn in range(3):
        s.q.copy_(torch.randn_like(s.q.float()))
        s.kn.copy_(torch.randn_like(s.kn.float()))
        s.parents = [some_tree(16, 10 * turn + b) for b in range(3)]
        s.parent.copy_(torch.tensor(s.parents, dtype=torch.int32))
        path[:, 0] = turn
        before = [s.kc[0].clone(), s.vc[0].clone(), s.n.clone(), s.out.clone()]
        s.ws.fill_(0xff)
        graph.replay()
        torch.cuda.synchronize()
        # what was kept: node `turn` of the second sequence in its first row
        n = before[2]
        assert torch.equal(s.n, n + accept[:, None])
        for h in range(2):
            at = int(n[1, h])
            assert torch.equal(s.kc[0][1, h, at], s.kn[1, h, turn]) and torch.equal(s.vc[0][1, h, at], s.vn[1, h, turn])
            for x, new in ((s.kc[0], s.kn), (s.vc[0], s.vn)):
                x[1, h, at] = new[1, h, 0] if families(s.parents[1])[0] else before[0][1, h, at]
        s.n.copy_(n)
        s.compare(before)
        s.n.copy_(n + accept[:, None])


def test_the_same_bits_every_time_and_on_two_streams(device):
    a, b = (Tree(device, [1000, 2000, 333], [some_tree(16, s + i) for i in range(3)], 32, 8, 128, W.WKV_BF16, 2100, seed=s) for s in (16, 17))
    first = []
    for s in (a, b):
        s.step()
        torch.cuda.synchronize()
        first.append(s.out.clone())
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(20):
        for s, st in zip((a, b), streams):
            with torch.cuda.stream(st):
                s.step()
    torch.cuda.synchronize()
    assert torch.equal(a.out, first[0]) and torch.equal(b.out, first[1])


def test_many_caches(device):
    # more (sequence, KV head) pairs than workgroups at a time: one range a cache, one launch
    counts = [17 + i % 50 for i in range(140)]
    Tree(device, counts, [some_tree(6, i) for i in range(140)], 16, 8, 64, W.WKV_BF16, 80, seed=18).check()


def accepted(path, want, T):
    out = []
    for x in path[:max(want, 0)]:
        if not 0 <= x < T or (out and x <= out[-1]):
            break
        out.append(x)
    return out


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("d,layout", [(64, "projection"), (128, "projection"), (128, "heads")])
@pytest.mark.parametrize("T", [1, 7, 64])
def test_acceptance(device, dtype, d, layout, T):
    r = random.Random(T)
    counts = [0, 50, 100 - T, 101 - T, -1, 20, 30]              # the fourth and fifth could not take a tree
    B, H, layers = len(counts), 2, 3
    s = Tree(device, counts, [some_tree(T, b) for b in range(B)], 4, H, d, dtype, 100, seed=T, layout=layout, layers=layers)
    for layer in range(layers):
        s.step(layer)
    paths = [sorted(r.sample(range(T), r.randrange(1, T + 1))) for _ in range(B)]
    paths = [p + [-1] * (T - len(p)) for p in paths]
    accept = [len([x for x in p if x >= 0]) for p in paths]
    accept[0] = T                                              # asks for more than the path has
    accept[5] = 0
    accept[6] = -5
    if T > 4:
        paths[1][:4] = [2, 5, 5, 6]                            # ascends for two nodes
        accept[1] = 4
    path, acc = (torch.tensor(x, dtype=torch.int32, device=device) for x in (paths, accept))
    was = [c.clone() for c in s.kc + s.vc]
    keep = W.TreeShape(batch=B, n_q_heads=4, n_kv_heads=H, head_dim=d, dtype=dtype, n_nodes=T, capacity=100, flags=W.WKV_DECODE_KEEP_COUNT,
                       cache_strides=(s.shape.c.cache_stride_b, s.shape.c.cache_stride_h, s.shape.c.cache_stride_t))
    n0 = s.n.clone()
    W.wkv_tree_accept(keep, s.kc[:1], s.vc[:1], path, acc, s.n)          # one layer, then the others and the count
    assert torch.equal(s.n, n0)
    W.wkv_tree_accept(s.shape, s.kc[1:], s.vc[1:], path, acc, s.n)
    torch.cuda.synchronize()
    for b in range(B):
        kept = accepted(paths[b], accept[b], T) if 0 <= counts[b] <= 100 - T else []
        assert (s.n[b] == counts[b] + len(kept)).all(), b
        for x, y in zip(s.kc + s.vc, was):
            for i, node in enumerate(kept):
                y[b, :, counts[b] + i] = y[b, :, counts[b] + node]          # (ascending: never a row that was written before)
    for x, y in zip(s.kc + s.vc, was):
        assert torch.equal(torch.isnan(x), torch.isnan(y)) and torch.equal(x.nan_to_num(), y.nan_to_num())


def test_offsets_past_32_bits(device):
    # 16 heads of 24576 rows of 128 fp32 channels, 192 MB each, 9 of them past 4 GiB from their sequence's first
    n, T, H = 16000, 4, 24
    cap = 500000
    s = None
    torch.cuda.empty_cache()
    kc, vc = (torch.zeros((1, H, cap, 128), dtype=torch.bfloat16, device=device) for _ in range(2))
    g = torch.Generator(device=device).manual_seed(19)
    far = H - 1
    kc[0, far, :n] = torch.randn((n, 128), device=device, generator=g).bfloat16()
    vc[0, far, :n] = torch.randn((n, 128), device=device, generator=g).bfloat16()
    assert far * cap * 128 > 2 ** 30
    q, kn, vn = (torch.randn((1, H, T, 128), device=device, generator=g).bfloat16() for _ in range(3))
    out = torch.zeros_like(q)
    counts = torch.full((1, H), n, dtype=torch.int32, device=device)
    shape = W.TreeShape(batch=1, n_q_heads=H, n_kv_heads=H, head_dim=128, dtype=W.WKV_BF16, n_nodes=T, capacity=cap)
    ws = torch.empty(W.wkv_tree_workspace_bytes(shape), dtype=torch.uint8, device=device)
    W.wkv_decode_tree(shape, q, kn, vn, torch.tensor([chain(T)], dtype=torch.int32, device=device), kc, vc, counts, out, ws)
    W.wkv_tree_accept(shape, [kc], [vc], torch.tensor([[1, 3, -1, -1]], dtype=torch.int32, device=device), torch.tensor([2], dtype=torch.int32, device=device), counts)
    for t in range(T):
        k = torch.cat([kc[0, far, :n], kn[0, far, :t + 1]]).double()
        v = torch.cat([vc[0, far, :n], vn[0, far, :t + 1]]).double()
        p = torch.softmax(q[0, far, t].double() @ k.t() / math.sqrt(128), -1)
        assert ((out[0, far, t].double() - p @ v).abs() <= 2.0 ** -8 * ((p @ v).abs() + p @ v.abs()) + 1e-3 * (p @ v.abs())).all()
    assert torch.equal(kc[0, far, n], kn[0, far, 1]) and torch.equal(vc[0, far, n + 1], vn[0, far, 3]) and (counts == n + 2).all()
    del kc, vc
    torch.cuda.empty_cache()
