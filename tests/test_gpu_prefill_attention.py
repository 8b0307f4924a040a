"""wkv_prefill_attention against softmax(q K^T scale) V in 64 bits, row by row, at the sizes, layouts and masks where it can go wrong."""
import math

import pytest
import torch

import paper_2503_17922_amd as W
from tests.test_attention_cut import SHAPES

pytestmark = pytest.mark.gpu

TYPES = {W.WKV_F32: torch.float32, W.WKV_BF16: torch.bfloat16, W.WKV_F16: torch.float16}


def attention(q, k, v, scale):
    """q [H, n, d], k, v [Hkv, m, d] in 64 bits: outputs, normalisers, and sum_j p_j |v_j|."""
    H, n, d = q.shape
    G, m = H // k.shape[0], k.shape[1]
    q, k, v = q.double(), k.double().repeat_interleave(G, 0), v.double().repeat_interleave(G, 0)
    s = q @ k.transpose(1, 2) * scale
    hidden = torch.arange(m, device=q.device)[None, :] > torch.arange(n, device=q.device)[:, None] + (m - n)
    s = s.masked_fill(hidden, -math.inf)
    lse = torch.logsumexp(s, -1)
    p = torch.where(hidden, torch.zeros_like(s), torch.exp(s - torch.where(lse == -math.inf, torch.zeros_like(lse), lse)[..., None]))
    return p @ v, lse, p @ v.abs()


def check(out, lse, q, k, v, scale, dtype, what=""):
    """A logit is a sum of d products in fp32: off by (d + 4) * 2^-24 * scale * |q| |k| at most (delta), so a probability by 2 delta;
    sums of m probabilities and products by m * 2^-24 each, exponents by 2^-22 together.  16-bit types round every probability
    by half a step, and every type the output once."""
    want, want_lse, size = attention(q, k, v, scale)
    n, m, d = q.shape[1], k.shape[1], q.shape[2]
    if n == 0:
        return
    t = TYPES[dtype]
    half = torch.finfo(t).eps / 2
    longest = float(k.double().norm(dim=-1).max()) if m else 0.0
    delta = (d + 4) * 2.0 ** -24 * scale * q.double().norm(dim=-1) * longest
    loose = 2 * delta + (2 * m + 8) * 2.0 ** -24
    tol = want.abs() * half + size * ((half if dtype != W.WKV_F32 else 0.0) + loose[..., None]) * (1 + half) + (2.0 ** -24 if dtype == W.WKV_F16 else 1e-38)
    err = (out.double() - want).abs()
    assert not (~(err <= tol)).any(), f"{what}: worst {float((err / tol).max())} of the tolerance"
    if lse is not None and lse.shape[-1]:
        r = min(n, lse.shape[-1])
        got, ref = lse[:, lse.shape[-1] - r:].double(), want_lse[:, n - r:]
        assert (lse[:, :lse.shape[-1] - r] == -math.inf).all(), what
        empty = ref == -math.inf
        assert torch.equal(got == -math.inf, empty), what
        e = torch.where(empty, torch.zeros_like(got), (got - ref).abs())
        lim = delta[:, n - r:] + (m + 8) * 2.0 ** -24 + torch.where(empty, torch.zeros_like(ref), ref.abs()) * 2.0 ** -22
        assert not (e > lim).any(), f"{what}: lse off by {float((e / lim).max())} of the tolerance"


def run(device, q_len, k_len, Hq, H, d, dtype, layout="padded", lse_rows=0, scale=0.0, seed=1, spread=1.0, junk=math.nan, change=None):
    g = torch.Generator(device=device).manual_seed(seed)
    t = TYPES[dtype]
    B = len(q_len)
    randn = lambda *shape: torch.randn(shape, device=device, generator=g)
    qs = [randn(Hq, n, d).mul(spread).to(t) for n in q_len]
    ks, vs = [randn(H, m, d).to(t) for m in k_len], [randn(H, m, d).to(t) for m in k_len]
    if change:
        change(qs, ks, vs)
    if layout == "packed":                   # [row, head, channel] with rows of nobody before, between and after
        gap = 3
        q_start = [gap + sum(q_len[:b]) + gap * b for b in range(B)]
        k_start = [2 + sum(k_len[:b]) + 5 * b for b in range(B)]
        Q, O = (torch.full((sum(q_len) + gap * (B + 2), Hq, d), x, dtype=t, device=device) for x in (junk, 7.0))
        K, V = (torch.full((sum(k_len) + 5 * (B + 2), H, d), junk, dtype=t, device=device) for _ in range(2))
        view = lambda x, start, n, b: x[start[b]:start[b] + n[b]].transpose(0, 1)
        kw = dict(q_start=q_start, k_start=k_start, q_strides=(0, d, Hq * d), kv_strides=(0, d, H * d))
        qv = lambda x, b: view(x, q_start, q_len, b)
        kv = lambda x, b: view(x, k_start, k_len, b)
    elif layout == "bthd":                   # token-major, as slices of one tensor
        rows, keys = max(max(q_len), 1), max(max(k_len), 1) + 2
        Q, O = (torch.full((B, rows, Hq, d), x, dtype=t, device=device) for x in (junk, 7.0))
        KV = torch.full((B, keys, 2 * H, d), junk, dtype=t, device=device)
        K, V = KV[:, :, :H], KV[:, :, H:]
        kw = dict(q_strides=(rows * Hq * d, d, Hq * d), kv_strides=(keys * 2 * H * d, d, 2 * H * d))
        qv = lambda x, b: x[b, :q_len[b]].transpose(0, 1)
        kv = lambda x, b: x[b, :k_len[b]].transpose(0, 1)
    else:
        rows, keys = max(max(q_len), 1), max(max(k_len), 1) + 9
        Q, O = (torch.full((B, Hq, rows, d), x, dtype=t, device=device) for x in (junk, 7.0))
        K, V = (torch.full((B, H, keys, d), junk, dtype=t, device=device) for _ in range(2))
        kw = dict(q_strides=(Hq * rows * d, rows * d, d), kv_strides=(H * keys * d, keys * d, d))
        qv = lambda x, b: x[b, :, :q_len[b]]
        kv = lambda x, b: x[b, :, :k_len[b]]
    for b in range(B):
        qv(Q, b).copy_(qs[b]); kv(K, b).copy_(ks[b]); kv(V, b).copy_(vs[b])
    shape = W.AttentionShape(q_len=q_len, k_len=k_len, n_q_heads=Hq, n_kv_heads=H, head_dim=d, dtype=dtype, scale=scale, lse_rows=lse_rows, **kw)
    lse = torch.full((B, Hq, lse_rows), 5.0, device=device) if lse_rows else None
    ws = torch.full((W.wkv_attention_workspace_bytes(shape),), 0xff, dtype=torch.uint8, device=device)
    call = lambda: W.wkv_prefill_attention(shape, Q, K, V, O, lse, ws)
    call()
    torch.cuda.synchronize()
    verify = lambda: [check(qv(O, b), lse[b] if lse_rows else None, qv(Q, b), kv(K, b), kv(V, b), scale or d ** -0.5, dtype, f"sequence {b}")
                      for b in range(B)]
    verify()
    rest = torch.ones_like(O, dtype=torch.bool)
    for b in range(B):
        qv(rest, b).fill_(False)
    assert (O[rest] == 7.0).all(), "rows of no sequence were written"
    return call, verify, Q, O, lse


LENGTHS = [1, 2, 7, 8, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 257, 500]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hq,H", [(4, 1), (3, 3), (7, 1), (16, 2)])
def test_prompts_of_all_lengths(device, dtype, d, Hq, H):
    for i in range(0, len(LENGTHS), 4):
        n = LENGTHS[i:i + 4]
        run(device, n, n, Hq, H, d, dtype, lse_rows=5, seed=i)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("layout", ["packed", "bthd"])
@pytest.mark.parametrize("d", [64, 128])
def test_layouts(device, dtype, layout, d):
    run(device, [130, 1, 64, 0, 300], [130, 1, 64, 0, 300], 6, 2, d, dtype, layout=layout, lse_rows=70)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("q_len,k_len", [([1], [1000]), ([1, 1, 1], [1, 64, 777]), ([5, 17], [700, 64 + 17]), ([100], [1100]), ([64, 3], [65, 515])])
def test_pieces_of_a_prompt(device, dtype, q_len, k_len):
    run(device, q_len, k_len, 8, 2, 128, dtype, lse_rows=4)
    run(device, q_len, k_len, 8, 1, 64, dtype, layout="packed", lse_rows=4)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("q_len,k_len", [([10], [3]), ([300], [1]), ([40, 130], [0, 90]), ([1], [0]), ([0, 0], [5, 0])])
def test_rows_without_keys(device, dtype, q_len, k_len):
    *_, O, lse = run(device, q_len, k_len, 4, 2, 128, dtype, lse_rows=max(max(q_len), 1))
    for b in range(len(q_len)):
        empty = max(q_len[b] - k_len[b], 0)
        assert (O[b, :, :empty] == 0).all()


@pytest.mark.parametrize("dtype", list(TYPES))
def test_logits_that_grow_along_the_keys(device, dtype):
    # every tile outgrows the ones before it, then the reverse; logits of several hundred
    def ramp(reverse):
        def change(qs, ks, vs):
            for q, k in zip(qs, ks):
                r = torch.linspace(0.1, 24.0, k.shape[1], device=k.device)[None, :, None]
                k.copy_(k.abs() * (r.flip(1) if reverse else r) * 0.5)
                q.copy_(q.abs())
        return change
    for reverse in (False, True):
        run(device, [400], [400], 4, 2, 128, dtype, lse_rows=400, change=ramp(reverse))


@pytest.mark.parametrize("dtype", [W.WKV_BF16, W.WKV_F32])
def test_logits_far_below_zero(device, dtype):
    def change(qs, ks, vs):
        for q, k in zip(qs, ks):
            q.fill_(40.0); k.copy_(-k.abs() * 40.0 - 40.0)              # logits of -18000 and less
    run(device, [150], [150], 2, 1, 64, dtype, lse_rows=150, change=change)


@pytest.mark.parametrize("scale", [1.0, 0.01])
def test_scale(device, scale):
    run(device, [90], [90], 4, 2, 64, W.WKV_BF16, scale=scale, lse_rows=90)


def test_one_key_is_its_value(device):
    call, verify, Q, O, lse = run(device, [1, 1], [1, 1], 4, 4, 128, W.WKV_F16, lse_rows=1)


@pytest.mark.parametrize("Hq,H,n", [(32, 8, 2000), (28, 4, 1501), (8, 8, 4097)])
def test_long_prompts(device, Hq, H, n):
    run(device, [n], [n], Hq, H, 128, W.WKV_BF16, lse_rows=32)


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(str(x) for x in s[:4]) + f"-{len(s[4])}x{s[4][0]}")
def test_every_cut_of_the_work(device, shape):
    Hq, H, d, dtype, q_len, k_len = shape
    run(device, q_len, k_len, Hq, H, d, dtype, lse_rows=7, seed=len(q_len))


def test_many_sequences(device):
    g = torch.Generator().manual_seed(9)
    n = torch.randint(0, 90, (64,), generator=g).tolist()
    m = [x + int(y) for x, y in zip(n, torch.randint(0, 300, (64,), generator=g))]
    run(device, n, m, 3, 1, 64, W.WKV_F16, layout="packed", lse_rows=3)
    run(device, n, m, 4, 2, 128, W.WKV_BF16, lse_rows=100)


def test_the_same_bits_again_and_replayed(device):
    call, verify, Q, O, lse = run(device, [700, 33], [700, 333], 8, 2, 128, W.WKV_BF16, lse_rows=8)
    first, first_lse = O.clone(), lse.clone()
    O.fill_(7.0); lse.fill_(0.0)
    call()
    torch.cuda.synchronize()
    assert torch.equal(O, first) and torch.equal(lse, first_lse)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        O.fill_(7.0)
        Q.nan_to_num_(0.0).mul_(0.5)
        graph.replay()
        torch.cuda.synchronize()
        verify()


def test_normalisers_as_the_score_call_takes_them(device):
    # token scores with the normalisers of this attention against those that the score call computes itself
    Hq, H, d, w, L = 8, 2, 128, 16, 900
    g = torch.Generator(device=device).manual_seed(3)
    q, k, v = (torch.randn((1, n, L, d), device=device, generator=g).bfloat16() for n in (Hq, H, H))
    out, lse = torch.zeros_like(q), torch.zeros((1, Hq, w), device=device)
    shape = W.AttentionShape(q_len=[L], n_q_heads=Hq, n_kv_heads=H, head_dim=d, dtype=W.WKV_BF16, lse_rows=w)
    W.wkv_prefill_attention(shape, q, k, v, out, lse, torch.empty(W.wkv_attention_workspace_bytes(shape), dtype=torch.uint8, device=device))
    p = W.Problem(n_q_heads=Hq, n_kv_heads=H, head_dim=d, w_obs=w, seq_len=[L], win=[8], top_p=[8], k_windows=[10], dtype=W.WKV_BF16)
    ws = torch.empty(W.wkv_workspace_bytes(p), dtype=torch.uint8, device=device)
    t = [torch.zeros((1, H, L - w), device=device) for _ in range(2)]
    q_obs = q[:, :, L - w:].contiguous()
    W.wkv_score(p, q_obs, k, lse, t[0], ws)
    W.wkv_score(p, q_obs, k, None, t[1], ws)
    assert torch.allclose(t[0], t[1], rtol=1e-4, atol=1e-9)
