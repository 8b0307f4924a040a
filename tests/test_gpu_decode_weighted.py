"""wkv_decode_step_weighted: the caches, counts and refusals of wkv_decode_step, outputs and weights against softmax(q K^T scale) in 64 bits."""
import pytest
import torch

import paper_2503_17922_amd as W

pytestmark = pytest.mark.gpu

TYPES = {W.WKV_F32: torch.float32, W.WKV_BF16: torch.bfloat16, W.WKV_F16: torch.float16}


class Caches:
    def __init__(self, device, counts, Hq, H, d, dtype, cap, seed=1, layout="bhtd", flags=0, spread=1.5):
        g = torch.Generator(device=device).manual_seed(seed)
        B, t = len(counts), TYPES[dtype]
        randn = lambda *s: torch.randn(s, device=device, generator=g)
        if layout == "bhtd":
            self.kc, self.vc = (randn(B, H, cap, d).to(t) for _ in range(2))
            strides = None
        else:
            self.kc, self.vc = (randn(B, cap, H, d).to(t).transpose(1, 2) for _ in range(2))
            strides = (cap * H * d, d, H * d)
        self.q, self.kn, self.vn = randn(B, Hq, d).mul(spread).to(t), randn(B, H, d).to(t), randn(B, H, d).to(t)
        self.n = torch.tensor(counts, dtype=torch.int32, device=device)
        if self.n.dim() == 1:
            self.n = self.n[:, None].repeat(1, H)
        self.weights = torch.rand((B, H, cap), device=device, generator=g) * 3
        self.tok = torch.randint(0, 10 ** 6, (B, H, cap), dtype=torch.int32, device=device, generator=g)
        self.at = torch.arange(B, device=device, dtype=torch.int32) + 2 ** 30
        self.out = torch.full((B, Hq, d), -5.0, device=device)
        self.shape = W.DecodeShape(batch=B, n_q_heads=Hq, n_kv_heads=H, head_dim=d, dtype=dtype, capacity=cap, cache_strides=strides, flags=flags)
        self.ws = torch.full((W.wkv_decode_weighted_workspace_bytes(self.shape),), 0xff, dtype=torch.uint8, device=device)
        self.cap, self.dtype, self.scale = cap, dtype, d ** -0.5

    def step(self, **kw):
        tok, at = kw.get("tok", self.tok), kw.get("at", self.at)
        W.wkv_decode_step_weighted(self.shape, self.q, self.kn, self.vn, self.kc, self.vc, self.n, self.weights, tok, at, self.out, self.ws)
        torch.cuda.synchronize()

    def check(self, keep_count=False, with_tok=True):
        before = {x: getattr(self, x).clone() for x in ("kc", "vc", "n", "weights", "tok")}
        plain = {x: before[x].clone(memory_format=torch.preserve_format) for x in ("kc", "vc", "n")}
        out = torch.full_like(self.out, 3.0)
        ws = torch.empty(W.wkv_decode_workspace_bytes(self.shape), dtype=torch.uint8, device=self.out.device)
        W.wkv_decode_step(self.shape, self.q, self.kn, self.vn, plain["kc"], plain["vc"], plain["n"], out, ws)
        self.step(**({} if with_tok else dict(tok=None, at=None)))
        # the step itself: the same rows, counts and refusals; the outputs below (a sum's order may be another)
        assert torch.equal(torch.isnan(self.out), torch.isnan(out))
        for x in plain:
            assert torch.equal(getattr(self, x), plain[x]), x
        want, tok, tol = before["weights"].double(), before["tok"], torch.zeros_like(before["weights"], dtype=torch.float64)
        B, H, cap = want.shape
        G = self.q.shape[1] // H
        d = self.q.shape[2]
        for b in range(B):
            for h in range(H):
                n = int(before["n"][b, h])
                if not 0 <= n < cap:
                    continue
                k = self.kc[b, h, :n + 1].double()
                q = self.q[b, h * G:(h + 1) * G].double()
                p = torch.softmax(q @ k.t() * self.scale, -1)
                want[b, h, n] = 0.0
                want[b, h, :n + 1] += p.sum(0)
                if with_tok:
                    tok[b, h, n] = self.at[b]
                # a logit is off by (d + 4) 2^-24 scale |q| |k|, a probability by twice that, its sum of n terms and the exponents by
                # (n + 8) 2^-24, the G additions and the one to the old weight by half a step of the result each
                delta = (d + 4) * 2.0 ** -24 * self.scale * q.norm(dim=-1) * k.norm(dim=-1).max()
                loose = 2 * delta[:, None] + (n + 16) * 2.0 ** -24
                tol[b, h, :n + 1] = (p * loose).sum(0) + (G + 1) * 2.0 ** -24 * want[b, h, :n + 1]
                v = self.vc[b, h, :n + 1].double()
                # (and a sum of n products by another (n + 16) 2^-24 of their magnitudes)
                assert ((self.out[b, h * G:(h + 1) * G].double() - p @ v).abs() <= (p @ v.abs()) * (loose + (n + 16) * 2.0 ** -24)).all(), (b, h, n)
        err = (self.weights.double() - want).abs()
        assert (err <= tol).all(), f"worst {float((err - tol).max())} past the tolerance"
        assert torch.equal(self.tok, tok)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hq,H", [(1, 1), (6, 3), (8, 2), (10, 2), (7, 1), (16, 2)])
def test_heads_and_types(device, dtype, d, Hq, H):
    c = Caches(device, [0, 1, 15, 63, 64, 200, 299], Hq, H, d, dtype, 301, seed=Hq)
    for _ in range(2):
        c.check()


@pytest.mark.parametrize("counts,cap", [([4128], 4400), ([20000], 20011), ([700] * 16, 1000), ([5, 3000, 128, 4127], 4128), ([4128] * 40, 4200)])
def test_cache_sizes(device, counts, cap):
    c = Caches(device, counts, 32, 8, 128, W.WKV_BF16, cap)
    c.check()


@pytest.mark.parametrize("dtype", [W.WKV_F16, W.WKV_F32])
def test_token_major_caches_and_counts_of_their_own(device, dtype):
    c = Caches(device, [[3, 100], [64, 0], [511, 17]], 8, 2, 64, dtype, 513, layout="bthd")
    for _ in range(3):
        c.check()


def test_full_caches_and_bad_counts_are_left_alone(device):
    c = Caches(device, [[50, -1], [49, 51], [2 ** 31 - 1, 7]], 8, 2, 128, W.WKV_BF16, 50)
    c.check()
    assert c.n.tolist() == [[50, -1], [50, 51], [2 ** 31 - 1, 8]]
    assert torch.isnan(c.out.view(3, 2, 4, 128)[0]).all() and not torch.isnan(c.out.view(3, 2, 4, 128)[1, 0]).any()


def test_without_positions_and_with_kept_counts(device):
    c = Caches(device, [77, 400], 8, 2, 128, W.WKV_BF16, 500, flags=W.WKV_DECODE_KEEP_COUNT)
    c.check(with_tok=False)
    assert c.n.tolist() == [[77, 77], [400, 400]]
    c.check()                                    # the same row again


@pytest.mark.parametrize("dtype", [W.WKV_BF16, W.WKV_F32])
def test_rows_of_infinite_logits_weigh_nothing(device, dtype):
    c = Caches(device, [40, 300], 4, 1, 64, dtype, 310)
    c.q.fill_(1.0)
    c.kc[0, 0, 5:30] = -float("inf")
    c.kc[1, 0] = -float("inf")
    before = c.weights.clone()
    c.step()
    assert torch.equal(c.weights[0, 0, 5:30], before[0, 0, 5:30]) and torch.equal(c.weights[1, 0, :300], before[1, 0, :300])
    assert abs(float(c.weights[1, 0, 300]) - 4.0) < 1e-5 and not torch.isnan(c.weights).any()
    # no row at all weighs anything: the weights stay, the new row's is 0
    c.kn.fill_(-float("inf"))
    c.n.fill_(300)
    before = c.weights.clone()
    c.step()
    assert torch.equal(c.weights[1, 0, :300], before[1, 0, :300]) and float(c.weights[1, 0, 300]) == 0.0


def test_captured_and_replayed(device):
    c = Caches(device, [100, 350], 8, 2, 128, W.WKV_BF16, 400)
    c.step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        W.wkv_decode_step_weighted(c.shape, c.q, c.kn, c.vn, c.kc, c.vc, c.n, c.weights, c.tok, c.at, c.out, c.ws)
    for step in range(3):
        c.q.copy_(torch.randn_like(c.q.float()))
        c.at += 1
        state = [getattr(c, x).clone() for x in ("kc", "vc", "n", "weights", "tok")]
        graph.replay()
        torch.cuda.synchronize()
        got = [getattr(c, x).clone() for x in ("kc", "vc", "n", "weights", "tok", "out")]
        for x, y in zip(("kc", "vc", "n", "weights", "tok"), state):
            getattr(c, x).copy_(y)
        c.step()
        for x, y in zip(("kc", "vc", "n", "weights", "tok", "out"), got):
            assert torch.equal(getattr(c, x), y), x


def check_whole(c, with_tok=True):
    """A step whose rows one workgroup takes, as (sequence, KV head) pairs fill the compute units: outputs, weights, caches and counts in 64 bits."""
    before = {x: getattr(c, x).clone(memory_format=torch.preserve_format) for x in ("kc", "vc", "n", "weights", "tok")}
    c.step(**({} if with_tok else dict(tok=None, at=None)))
    B, H, cap = c.weights.shape
    G, d = c.q.shape[1] // H, c.q.shape[2]
    assert B * H >= 224 and cap <= 20224 // G // 16 * 16
    out = c.out.view(B, H, G, d)
    want = {x: before[x] for x in before}
    for b in range(B):
        for h in range(H):
            n = int(before["n"][b, h])
            if not 0 <= n < cap:
                assert torch.isnan(out[b, h]).all()
                continue
            want["kc"][b, h, n], want["vc"][b, h, n], want["n"][b, h] = c.kn[b, h], c.vn[b, h], n + 1
            if with_tok:
                want["tok"][b, h, n] = c.at[b]
            q, k, v = c.q[b, h * G:(h + 1) * G].double(), want["kc"][b, h, :n + 1].double(), want["vc"][b, h, :n + 1].double()
            p = torch.softmax(q @ k.t() * c.scale, -1)
            # a logit is off by (d + 4) 2^-24 scale |q| |k|, a probability by twice that and, with the sum of n terms and the exponents, (n + 16) 2^-24; sums of
            # products by as much again, the additions to a weight by half a step of the result each
            delta = (d + 4) * 2.0 ** -24 * c.scale * q.norm(dim=-1) * k.norm(dim=-1).max()
            loose = 2 * delta[:, None] + (n + 16) * 2.0 ** -24
            assert ((out[b, h].double() - p @ v).abs() <= (p @ v.abs()) * (loose + (n + 16) * 2.0 ** -24)).all(), (b, h, n)
            w = before["weights"][b, h, :n + 1].double()
            w[n] = 0.0
            w += p.sum(0)
            tol = (p * loose).sum(0) + (G + 1) * 2.0 ** -24 * w
            assert ((c.weights[b, h, :n + 1].double() - w).abs() <= tol).all(), (b, h, n)
            assert torch.equal(c.weights[b, h, n + 1:], before["weights"][b, h, n + 1:])
    for x in ("kc", "vc", "n", "tok"):
        assert torch.equal(getattr(c, x), want[x]), x


@pytest.mark.parametrize("dtype", [W.WKV_BF16, W.WKV_F16])
@pytest.mark.parametrize("B,Hq,H,d,cap,layout", [(64, 16, 4, 128, 300, "bhtd"), (7, 32, 32, 128, 700, "bthd"), (52, 64, 8, 64, 200, "bhtd"), (56, 24, 8, 128, 130, "bthd"),
                                                 (60, 20, 4, 64, 4032, "bhtd"), (56, 16, 4, 128, 5056, "bhtd"), (128, 14, 2, 64, 17, "bthd"), (7, 64, 32, 64, 10112, "bhtd")])
def test_a_workgroup_a_cache(device, dtype, B, Hq, H, d, cap, layout):
    g = torch.Generator().manual_seed(cap)
    counts = torch.randint(0, cap, (B, H), generator=g)
    counts.view(-1)[:9] = torch.tensor([0, 1, 15, 16, cap - 1, cap, -1, cap + 5, 2 ** 31 - 1])
    c = Caches(device, counts.tolist(), Hq, H, d, dtype, cap, layout=layout)
    check_whole(c)
    check_whole(c, with_tok=False)


def test_a_workgroup_a_cache_with_kept_counts_and_infinite_logits(device):
    c = Caches(device, [100] * 56, 16, 4, 128, W.WKV_BF16, 128, flags=W.WKV_DECODE_KEEP_COUNT)
    before = c.weights.clone()
    c.q.fill_(1.0)
    c.kc[:28, :, 5:30] = -float("inf")
    c.kc[28:] = -float("inf")
    c.step()
    assert (c.n == 100).all() and not torch.isnan(c.weights).any()
    assert torch.equal(c.weights[:28, :, 5:30], before[:28, :, 5:30]) and torch.equal(c.weights[28:, :, :100], before[28:, :, :100])
    assert (c.weights[:28, :, :5] > before[:28, :, :5]).any() and ((c.weights[28:, :, 100] - 4.0).abs() < 1e-5).all()
    assert torch.equal(c.out[28:].view(28, 4, 4, 128), c.vn[28:, :, None].float().expand(28, 4, 4, 128))
    c.kn.fill_(-float("inf"))
    before = c.weights.clone()
    c.step()
    assert torch.equal(c.weights[28:, :, :100], before[28:, :, :100]) and (c.weights[28:, :, 100] == 0).all()


def test_a_workgroup_a_cache_captured_and_replayed(device):
    c = Caches(device, [200 + i for i in range(64)], 16, 4, 128, W.WKV_BF16, 300)
    names = ("kc", "vc", "n", "weights", "tok", "out")
    c.step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        W.wkv_decode_step_weighted(c.shape, c.q, c.kn, c.vn, c.kc, c.vc, c.n, c.weights, c.tok, c.at, c.out, c.ws)
    for step in range(3):
        c.q.copy_(torch.randn_like(c.q.float()))
        c.at += 1
        state = [getattr(c, x).clone() for x in names]
        graph.replay()
        torch.cuda.synchronize()
        got = [getattr(c, x).clone() for x in names]
        for x, y in zip(names, state):
            getattr(c, x).copy_(y)
        check_whole(c)
        for x, y in zip(names, got):
            assert torch.equal(getattr(c, x), y), x


@pytest.mark.parametrize("cap", [1, 16, 17, 128, 129, 256, 257])
@pytest.mark.parametrize("dtype,Hq,H,d", [(W.WKV_BF16, 8, 2, 128), (W.WKV_F16, 3, 1, 128), (W.WKV_BF16, 8, 1, 64), (W.WKV_F16, 2, 2, 64), (W.WKV_BF16, 16, 2, 128)])
def test_short_caches(device, dtype, Hq, H, d, cap):
    counts = sorted({0, cap // 2, max(cap - 2, 0), cap - 1, cap})
    c = Caches(device, counts, Hq, H, d, dtype, cap)
    for _ in range(2):
        c.check()
