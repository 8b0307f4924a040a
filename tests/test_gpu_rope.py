"""wkv_rope against the rotation in 64 bits, at the layouts, types and positions where it can go wrong."""
import math

import pytest
import torch

import paper_2503_17922_amd as W

pytestmark = pytest.mark.gpu

TYPES = {W.WKV_F32: torch.float32, W.WKV_BF16: torch.bfloat16, W.WKV_F16: torch.float16}


def turned(x, pos, inv, amplitude, interleaved, inverse=False):
    """x [B, H, T, d] in 64 bits, pairs of the first 2 * len(inv) channels turned; and the sum of a pair's magnitudes."""
    r = 2 * len(inv)
    i = torch.arange(r // 2, device=x.device)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + r // 2)
    angle = pos.double()[:, None, :, None] * torch.tensor(inv, dtype=torch.float64, device=x.device)
    c, s = amplitude * angle.cos(), amplitude * angle.sin() * (-1 if inverse else 1)
    y, size = x.double().clone(), x.double().abs()
    x0, x1 = y[..., a].clone(), y[..., b].clone()
    y[..., a], y[..., b] = x0 * c - x1 * s, x1 * c + x0 * s
    size[..., a] = size[..., b] = (x0.abs() + x1.abs()) * abs(amplitude)
    return y, size


def check(got, want, size, dtype):
    """The angle is off by up to half a step of a float of at most pi (2^-24 * pi), sine and cosine by two steps, each product
    and the sum by half a step: less than 2^-21 of the pair's magnitudes; then one rounding to the type."""
    t = TYPES[dtype]
    half = torch.finfo(t).eps / 2
    tol = size * 2.0 ** -21 * (1 + half) + want.abs() * half + (2.0 ** -25 if t == torch.float16 else 1e-45)
    bad = (got.double() - want).abs() > tol
    assert not bad.any(), f"{int(bad.sum())} elements off, worst {float(((got.double() - want).abs() / tol).max())} of the tolerance"


def make(B, T, Hq, H, d, dtype, device, seed):
    g = torch.Generator(device=device).manual_seed(seed)
    rows = torch.randn((B, T, Hq + 2 * H, d), device=device, generator=g).to(TYPES[dtype])
    return rows


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("d,rotary", [(128, 128), (128, 64), (128, 16), (128, 112), (64, 64), (64, 32), (64, 16), (64, 48)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_layouts(device, dtype, d, rotary, interleaved):
    B, T, Hq, H = 2, 37, 7, 3
    rows = make(B, T, Hq, H, d, dtype, device, 1)
    inv, amp = W.wkv_rope_frequencies(rotary, 10000.0)
    pos = torch.randint(0, 40000, (B, T), dtype=torch.int32, device=device, generator=torch.Generator(device=device).manual_seed(2))
    pos[0, 5] = pos[1, 36] = -1                                  # padding
    n = Hq + 2 * H
    cap = T + 5
    shape = W.RopeShape(batch=B, n_tokens=T, n_q_heads=Hq, n_kv_heads=H, head_dim=d, dtype=dtype, inv_freq=inv, amplitude=amp,
                        interleaved=interleaved, q_strides=(T * n * d, d, n * d), k_strides=(T * n * d, d, n * d),
                        q_out_strides=(T * Hq * d, d, Hq * d), k_out_strides=(H * cap * d, cap * d, d))
    q_out = torch.full((B, T, Hq, d), 7.0, dtype=TYPES[dtype], device=device)
    cache = torch.full((B, H, cap, d), 7.0, dtype=TYPES[dtype], device=device)
    before = rows.clone()
    W.wkv_rope(shape, pos, rows, q_out, rows[:, :, Hq:], cache)
    torch.cuda.synchronize()
    assert torch.equal(rows, before)
    for x, got in ((rows[:, :, :Hq], q_out.transpose(1, 2)), (rows[:, :, Hq:Hq + H], cache[:, :, :T])):
        want, size = turned(x.transpose(1, 2), pos, inv, amp, interleaved)
        padding = (pos < 0)[:, None, :, None].expand_as(want)
        assert (got[padding] == 7.0).all(), "rows without a position are left alone"
        check(got[~padding], want[~padding], size[~padding], dtype)
        copied = x.transpose(1, 2)[..., rotary:]
        assert torch.equal(torch.where(padding[..., rotary:], copied, got[..., rotary:]), copied), "channels past the rotary ones"
    assert (cache[:, :, T:] == 7.0).all()


@pytest.mark.parametrize("B,T,Hq,H", [(1, 1, 1, 1), (64, 1, 32, 8), (3, 1, 28, 4), (1, 5, 0, 2), (2, 3, 9, 0), (1, 4099, 3, 1), (1, 9000, 1, 1)])
def test_sizes_from_one_token_to_long_ones(device, B, T, Hq, H):
    d, dtype = 128, W.WKV_BF16
    inv, amp = W.wkv_rope_frequencies(d, 500000.0)
    g = torch.Generator(device=device).manual_seed(3)
    q = torch.randn((B, max(Hq, 1), T, d), device=device, generator=g).bfloat16()
    k = torch.randn((B, max(H, 1), T, d), device=device, generator=g).bfloat16()
    pos = (torch.arange(T, device=device, dtype=torch.int32) + 5).repeat(B, 1)
    qo, ko = torch.zeros_like(q), torch.zeros_like(k)
    shape = W.RopeShape(batch=B, n_tokens=T, n_q_heads=Hq, n_kv_heads=H, head_dim=d, dtype=dtype, inv_freq=inv)
    W.wkv_rope(shape, pos, q if Hq else None, qo if Hq else None, k if H else None, ko if H else None)
    for x, got, heads in ((q, qo, Hq), (k, ko, H)):
        if heads:
            check(got, *turned(x, pos, inv, 1.0, False), dtype)


def test_far_positions(device):
    # the angle in turns is exact for every position: 2^31 - 1 is turned as well as 0
    inv, _ = W.wkv_rope_frequencies(128, 10000.0)
    pos = torch.tensor([[0, 1, 2 ** 20, 2 ** 24 + 1, 2 ** 30 + 3, 2 ** 31 - 1]], dtype=torch.int32, device=device)
    x = torch.randn((1, 2, 6, 128), device=device, generator=torch.Generator(device=device).manual_seed(4))
    got = torch.zeros_like(x)
    W.wkv_rope(W.RopeShape(batch=1, n_tokens=6, n_q_heads=2, n_kv_heads=0, head_dim=128, dtype=W.WKV_F32, inv_freq=inv), pos, x, got, None, None)
    # (the oracle in 80 bits on the host: 64 bits leave 2^31 * 2^-53 of a radian)
    import numpy as np
    angle = pos[0].cpu().numpy().astype(np.longdouble)[:, None] * np.array(inv, dtype=np.longdouble)
    c, s = (torch.from_numpy(f(angle).astype(np.float64)).to(device) for f in (np.cos, np.sin))
    x0, x1 = x[..., :64].double(), x[..., 64:].double()
    check(got, torch.cat([x0 * c - x1 * s, x1 * c + x0 * s], -1), (x0.abs() + x1.abs()).repeat(1, 1, 1, 2), W.WKV_F32)


@pytest.mark.parametrize("interleaved", [False, True])
def test_in_place_and_back(device, interleaved):
    inv, amp = W.wkv_rope_frequencies(64, 10000.0, W.WKV_ROPE_PARTS, 4.0, 4096)
    x = torch.randn((2, 3, 11, 64), device=device, generator=torch.Generator(device=device).manual_seed(5))
    pos = torch.arange(22, device=device, dtype=torch.int32).view(2, 11) * 977
    kw = dict(batch=2, n_tokens=11, n_q_heads=3, n_kv_heads=3, head_dim=64, dtype=W.WKV_F32, inv_freq=inv, interleaved=interleaved)
    q, k = x.clone(), x.clone()
    W.wkv_rope(W.RopeShape(amplitude=amp, **kw), pos, q, q, k, k)
    want, size = turned(x, pos, inv, amp, interleaved)
    check(q, want, size, W.WKV_F32)
    assert torch.equal(q, k)
    W.wkv_rope(W.RopeShape(amplitude=1.0 / amp, inverse=True, **kw), pos, q, q, k, k)
    # twice the error of a turn, the second one of turned pairs (at most sqrt(2) the magnitudes)
    assert ((q - x).abs() <= 3 * size * 2.0 ** -21).all()


def test_the_inverse_is_the_gradient(device):
    # y = R x: dL/dx = R^T dL/dy, against differences of L in 64 bits
    inv, amp = W.wkv_rope_frequencies(32, 10000.0)
    g = torch.Generator(device=device).manual_seed(6)
    x, dy = (torch.randn((1, 1, 3, 64), device=device, generator=g) for _ in range(2))
    pos = torch.tensor([[3, 500, 70000]], dtype=torch.int32, device=device)
    dx = torch.zeros_like(dy)
    W.wkv_rope(W.RopeShape(batch=1, n_tokens=3, n_q_heads=1, n_kv_heads=0, head_dim=64, dtype=W.WKV_F32, inv_freq=inv, amplitude=1.5, inverse=True),
               pos, dy, dx, None, None)
    loss = lambda z: (turned(z, pos, inv, 1.5, False)[0] * dy.double()).sum()
    h = 2.0 ** -10
    for t in range(3):
        for c in (0, 5, 16, 31, 32, 63):
            e = torch.zeros_like(x, dtype=torch.float64)
            e[0, 0, t, c] = h
            difference = (loss(x.double() + e) - loss(x.double() - e)) / (2 * h)      # (linear: exact up to rounding)
            assert abs(float(difference) - float(dx[0, 0, t, c])) <= 1e-5 * float(dy.abs().max())


def test_captured_and_replayed(device):
    inv, _ = W.wkv_rope_frequencies(128, 10000.0)
    shape = W.RopeShape(batch=4, n_tokens=1, n_q_heads=8, n_kv_heads=2, head_dim=128, dtype=W.WKV_BF16, inv_freq=inv)
    q, k = torch.randn((4, 8, 1, 128), device=device).bfloat16(), torch.randn((4, 2, 1, 128), device=device).bfloat16()
    qo, ko = torch.zeros_like(q), torch.zeros_like(k)
    pos = torch.tensor([[1], [2], [3], [4]], dtype=torch.int32, device=device)
    W.wkv_rope(shape, pos, q, qo, k, ko)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        W.wkv_rope(shape, pos, q, qo, k, ko)
    for step in range(3):
        pos += 1000 * step
        q.copy_(torch.randn_like(q.float()).bfloat16())
        graph.replay()
        torch.cuda.synchronize()
        check(qo, *turned(q, pos, inv, 1.0, False), W.WKV_BF16)
        check(ko, *turned(k, pos, inv, 1.0, False), W.WKV_BF16)


def test_infinities_and_nan_stay_in_their_pairs(device):
    inv, _ = W.wkv_rope_frequencies(64, 10000.0)
    x = torch.ones((1, 1, 2, 64), device=device)
    x[0, 0, 0, 3], x[0, 0, 1, 60] = math.nan, math.inf
    y = torch.zeros_like(x)
    W.wkv_rope(W.RopeShape(batch=1, n_tokens=2, n_q_heads=1, n_kv_heads=0, head_dim=64, dtype=W.WKV_F32, inv_freq=inv),
               torch.tensor([[7, 8]], dtype=torch.int32, device=device), x, y, None, None)
    assert (~torch.isfinite(y)).nonzero().tolist() == [[0, 0, 0, 3], [0, 0, 0, 35], [0, 0, 1, 28], [0, 0, 1, 60]]
