"""The operators around the compression where tensors are large or calls run side by side: offsets past 32 bits against the same call on compact
tensors, bit for bit, and calls on two other streams against the same calls one after the other."""
import pytest
import torch

import paper_2503_17922_amd as W
from tests.test_gpu_decode_weighted import Caches
from tests.test_gpu_evict import State
from tests.test_gpu_prefill_attention import check as check_attention

pytestmark = pytest.mark.gpu

FAR = (1 << 32) + 4096                    # elements: past 32 bits as a number of elements, of bytes twice over


@pytest.fixture(autouse=True)
def give_memory_back():
    yield
    torch.cuda.empty_cache()


def spread_out(x, strides, first=0):
    """A copy of x with these strides (of all axes but the last), from element `first` on; what lies between is not initialised."""
    size = first + sum((n - 1) * s for n, s in zip(x.shape, strides)) + x.shape[-1]
    y = torch.empty(size, dtype=x.dtype, device=x.device).as_strided(x.shape, (*strides, 1), first)
    return y.copy_(x)


@pytest.mark.parametrize("axis", ["batch", "head", "token"])
def test_rope(device, axis):
    B, H, T, d = 2, 3, 3, 64
    g = torch.Generator(device=device).manual_seed(1)
    x, k = (torch.randn((B, H, T, d), device=device, generator=g).bfloat16() for _ in range(2))
    pos = torch.randint(0, 1 << 20, (B, T), dtype=torch.int32, device=device, generator=g)
    far = dict(batch=(FAR, T * d, d), head=(T * d, FAR // 2, d), token=(T * FAR // 2, d, FAR // 2))[axis]
    near = (H * T * d, T * d, d)
    inv, _ = W.wkv_rope_frequencies(d, 10000.0)
    kw = dict(batch=B, n_tokens=T, n_q_heads=H, n_kv_heads=H, head_dim=d, dtype=W.WKV_BF16, inv_freq=inv)
    want = torch.empty_like(x), torch.empty_like(k)
    W.wkv_rope(W.RopeShape(**kw), pos, x, want[0], k, want[1])
    # the queries read far apart and written together, the keys the other way round
    src, dst = spread_out(x, far), spread_out(torch.zeros_like(k), far)
    out = torch.empty_like(x)
    W.wkv_rope(W.RopeShape(q_strides=far, q_out_strides=near, k_strides=near, k_out_strides=far, **kw), pos, src, out, k, dst)
    assert torch.equal(out, want[0]) and torch.equal(dst, want[1])


@pytest.mark.parametrize("far", ["heads", "first row", "batch"])
@pytest.mark.parametrize("dtype", [W.WKV_BF16, W.WKV_F32])
def test_attention(device, far, dtype):
    B, H, n, d = 2, 2, 300, 64
    t = torch.bfloat16 if dtype == W.WKV_BF16 else torch.float32
    away = FAR // 4 if dtype == W.WKV_F32 else FAR // 2 + 64          # elements, in either type past 32 bits of bytes
    g = torch.Generator(device=device).manual_seed(2)
    q, k, v = (torch.randn((B, H, n, d), device=device, generator=g).to(t) for _ in range(3))
    first = [away // d, away // d] if far == "first row" else None
    strides = dict(heads=(n * d, away, d), batch=(away, n * d, d)).get(far, (H * n * d, n * d, d))
    lay = lambda x: spread_out(x, strides, first[0] * d if first else 0)
    whole = lambda x: x.as_strided((x.untyped_storage().size() // x.element_size(),), (1,), 0)      # from the start of its memory
    kw = dict(q_len=[n] * B, n_q_heads=H, n_kv_heads=H, head_dim=d, dtype=dtype, lse_rows=5)
    shape = W.AttentionShape(q_strides=strides, kv_strides=strides, q_start=first, k_start=first, **kw)
    Q, K, V, out = lay(q), lay(k), lay(v), lay(torch.zeros_like(q))
    lse = torch.empty((B, H, 5), device=device)
    ws = torch.empty(W.wkv_attention_workspace_bytes(shape), dtype=torch.uint8, device=device)
    W.wkv_prefill_attention(shape, *[whole(x) for x in (Q, K, V, out)], lse, ws)
    near, near_lse = torch.empty_like(q), torch.empty_like(lse)
    W.wkv_prefill_attention(W.AttentionShape(**kw), q, k, v, near, near_lse, ws)
    assert torch.equal(out, near) and torch.equal(lse, near_lse)
    for b in range(B):
        check_attention(out[b], lse[b], q[b], k[b], v[b], d ** -0.5, dtype)


def test_attention_over_keys_far_apart(device):
    n, d, t = 150, 128, torch.float16
    apart = (2 ** 31 - 1) // (2 * 64) // 8 * 8                # the largest token stride there is: 150 rows span 5 GB
    g = torch.Generator(device=device).manual_seed(3)
    q, k, v = (torch.randn((1, 1, n, d), device=device, generator=g).to(t) for _ in range(3))
    far = (n * apart, n * apart, apart)
    kw = dict(q_len=[n], n_q_heads=1, n_kv_heads=1, head_dim=d, dtype=W.WKV_F16)
    shape = W.AttentionShape(q_strides=far, kv_strides=far, **kw)
    ws = torch.empty(W.wkv_attention_workspace_bytes(shape), dtype=torch.uint8, device=device)
    out, near = spread_out(torch.zeros_like(q), far), torch.empty_like(q)
    W.wkv_prefill_attention(shape, spread_out(q, far), spread_out(k, far), spread_out(v, far), out, None, ws)
    W.wkv_prefill_attention(W.AttentionShape(**kw), q, k, v, near, None, ws)
    assert torch.equal(out, near)
    check_attention(out[0], None, q[0], k[0], v[0], d ** -0.5, W.WKV_F16)


@pytest.mark.parametrize("axis", ["head", "token"])
def test_weighted_step_and_eviction(device, axis):
    """Caches whose rows lie far apart, and long arrays of weights: the last (sequence, KV head) begins past 2^31 elements."""
    B, H, d, n, cap = 3, 3, 64, 40, 1 << 28
    near = Caches(device, [n] * B, H, H, d, W.WKV_BF16, n + 2, seed=4)
    strides = dict(head=(H * FAR // 2, FAR // 2, d), token=((n + 2) * FAR // 64, d, FAR // 64))[axis]
    kc, vc = spread_out(near.kc, strides), spread_out(near.vc, strides)
    shape = W.DecodeShape(batch=B, n_q_heads=H, n_kv_heads=H, head_dim=d, dtype=W.WKV_BF16, capacity=cap, cache_strides=strides)
    weights, tok = torch.empty((B, H, cap), device=device), torch.empty((B, H, cap), dtype=torch.int32, device=device)
    weights[:, :, :n], tok[:, :, :n] = near.weights[:, :, :n], near.tok[:, :, :n]
    count, out = near.n.clone(), torch.empty_like(near.out)
    ws = torch.empty(max(W.wkv_decode_weighted_workspace_bytes(shape), W.wkv_evict_workspace_bytes(shape)), dtype=torch.uint8, device=device)
    W.wkv_decode_step_weighted(shape, near.q, near.kn, near.vn, kc, vc, count, weights, tok, near.at, out, ws)
    near.check()
    # (the ranges of the keys differ with the capacity, so the sums' order does: a step of 2^-24 for each of 41 rows, twice)
    assert torch.equal(count, near.n) and torch.equal(kc, near.kc) and torch.equal(vc, near.vc) and torch.equal(tok[:, :, :n + 1], near.tok[:, :, :n + 1])
    rest = 2 * (n + 16) * 2.0 ** -24
    assert ((weights[:, :, :n + 1] - near.weights[:, :, :n + 1]).abs() <= rest * (near.weights[:, :, :n + 1] + 1)).all()
    size = near.vc[:, :, :n + 1].abs().amax((2, 3))[..., None]
    assert ((out - near.out).abs() <= 2 * (2 * 2.0 ** -9 + rest) * size).all()          # (probabilities in bf16: half a step each)
    # the eviction, by the same weights
    near.weights[:, :, :n + 1] = weights[:, :, :n + 1]
    keep = torch.full((B, H), n // 2, dtype=torch.int32, device=device)
    small_ws = torch.empty(W.wkv_evict_workspace_bytes(near.shape), dtype=torch.uint8, device=device)
    W.wkv_cache_evict(near.shape, [near.kc], [near.vc], near.weights, near.tok, near.n, keep, 3, small_ws)
    W.wkv_cache_evict(shape, [kc], [vc], weights, tok, count, keep, 3, ws)
    assert torch.equal(count, near.n) and torch.equal(kc, near.kc) and torch.equal(vc, near.vc)
    assert torch.equal(weights[:, :, :n + 1], near.weights[:, :, :n + 1]) and torch.equal(tok[:, :, :n + 1], near.tok[:, :, :n + 1])


def test_two_calls_at_once(device):
    """Every operator on two other streams at a time, each call with a workspace of its own."""
    t, B, H, d = torch.bfloat16, 2, 2, 128
    g = torch.Generator(device=device).manual_seed(5)
    inv, _ = W.wkv_rope_frequencies(d, 10000.0)

    class One:
        def __init__(self, seed, n, past):
            self.x, self.k, self.v = (torch.randn((B, m, n + past, d), device=device, generator=g).to(t) for m in (4, H, H))
            self.pos = torch.randint(0, 100000, (B, n + past), dtype=torch.int32, device=device, generator=g)
            self.rope = W.RopeShape(batch=B, n_tokens=n + past, n_q_heads=4, n_kv_heads=H, head_dim=d, dtype=W.WKV_BF16, inv_freq=inv)
            self.att = W.AttentionShape(q_len=[n, n // 2], k_len=[n + past, n], n_q_heads=4, n_kv_heads=H, head_dim=d, dtype=W.WKV_BF16, lse_rows=4,
                                        q_strides=(4 * (n + past) * d, (n + past) * d, d), kv_strides=(H * (n + past) * d, (n + past) * d, d))
            self.ws = torch.empty(W.wkv_attention_workspace_bytes(self.att), dtype=torch.uint8, device=device)
            self.decode = Caches(device, [n, n // 3], 4, H, d, W.WKV_BF16, n + 5, seed=seed)
            self.evict = State(device, [n, n - 7], n // 2, 8, seed=seed)
            self.firsts = [y.clone() for y in self.state()]
            self.q, self.kr, self.out = torch.zeros_like(self.x), torch.zeros_like(self.k), torch.zeros_like(self.x)
            self.lse = torch.zeros((B, 4, 4), device=device)

        def state(self):
            c, e = self.decode, self.evict
            return [c.kc, c.vc, c.n, c.weights, c.tok] + e.tensors() + [e.n]

        def reset(self):
            for y, first in zip(self.state(), self.firsts):
                y.copy_(first)
            for y in (self.q, self.kr, self.out, self.lse):
                y.zero_()

        def run(self):
            W.wkv_rope(self.rope, self.pos, self.x, self.q, self.k, self.kr)
            W.wkv_prefill_attention(self.att, self.q, self.kr, self.v, self.out, self.lse, self.ws)
            c = self.decode
            W.wkv_decode_step_weighted(c.shape, c.q, c.kn, c.vn, c.kc, c.vc, c.n, c.weights, c.tok, c.at, c.out, c.ws)
            self.evict.call()

        def results(self):
            return [y.clone() for y in self.state() + [self.q, self.kr, self.out, self.lse, self.decode.out]]

    ones = [One(6, 900, 0), One(7, 40, 3000)]
    want = []
    for one in ones:
        one.run()
        want.append(one.results())
    for turn in range(3):
        for one in ones:
            one.reset()
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream() for _ in ones]
        for one, stream in zip(ones, streams):
            with torch.cuda.stream(stream):
                one.run()
        torch.cuda.synchronize()
        for i, (one, w) in enumerate(zip(ones, want)):
            for j, (x, y) in enumerate(zip(one.results(), w)):
                assert torch.equal(x, y), f"call {i}, result {j}"
