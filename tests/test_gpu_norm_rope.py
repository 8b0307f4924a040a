"""wkv_norm_rope against the norm and the rotation in 64 bits, at the layouts, types, axes and positions where it can go wrong."""
import math

import pytest
import torch

import paper_2503_17922_amd as W

pytestmark = pytest.mark.gpu

TYPES = {W.WKV_F32: torch.float32, W.WKV_BF16: torch.bfloat16, W.WKV_F16: torch.float16}


def expected(x, weight, pos, inv, axis, eps, amplitude, interleaved):
    """x [B, H, T, d] in 64 bits, normalised and turned; and the magnitudes that an error is measured by."""
    y = x.double()
    if weight is not None:
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps) * weight.double()
    else:
        y = y.clone()
    r = 2 * len(inv)
    i = torch.arange(r // 2, device=x.device)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + r // 2)
    where = pos.double()[..., torch.tensor(axis, device=x.device)]                    # [B, T, pairs]
    angle = (where * torch.tensor(inv, dtype=torch.float64, device=x.device))[:, None]
    c, s = amplitude * angle.cos(), amplitude * angle.sin()
    size = y.abs()
    y0, y1 = y[..., a].clone(), y[..., b].clone()
    y[..., a], y[..., b] = y0 * c - y1 * s, y1 * c + y0 * s
    size[..., a] = size[..., b] = (y0.abs() + y1.abs()) * abs(amplitude)
    return y, size


def check(got, want, size, dtype):
    """Sums of 128 squares in fp32 are off by at most 24 steps of 2^-24 (16 in a lane, 3 across, the product with 1 / d and the sum with
    eps), their root by half of that and its own step, the reciprocal and the two products by one each: 16 * 2^-24 = 2^-20 in all.
    The rotation adds 2^-21 of a pair's magnitudes, as for the rotation alone; then one rounding to the type."""
    t = TYPES[dtype]
    half = torch.finfo(t).eps / 2
    tol = size * (2.0 ** -20 + 2.0 ** -21) * (1 + half) + want.abs() * half + (2.0 ** -25 if t == torch.float16 else 1e-45)
    bad = ~((got.double() - want).abs() <= tol)
    assert not bad.any(), f"{int(bad.sum())} elements off, worst {float(((got.double() - want).abs() / tol).max())} of the tolerance"


def weights(d, dtype, device, seed):
    g = torch.Generator(device=device).manual_seed(seed)
    return (1 + 0.5 * torch.randn(d, device=device, generator=g)).to(TYPES[dtype])


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("d,rotary", [(128, 128), (128, 64), (128, 16), (128, 112), (64, 64), (64, 16), (64, 48)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("axes", [1, 3])
def test_layouts(device, dtype, d, rotary, interleaved, axes):
    B, T, Hq, H, eps = 2, 37, 7, 3, 1e-5
    g = torch.Generator(device=device).manual_seed(1)
    n, cap = Hq + 2 * H, T + 5
    rows = (torch.randn((B, T, n, d), device=device, generator=g) * torch.exp(torch.randn((B, T, n, 1), device=device, generator=g))).to(TYPES[dtype])
    inv, amp = W.wkv_rope_frequencies(rotary, 10000.0, W.WKV_ROPE_PARTS, 4.0, 4096)
    axis = [(5 * i + i // 3) % axes for i in range(rotary // 2)]
    pos = torch.randint(0, 40000, (B, T, axes), dtype=torch.int32, device=device, generator=g)
    pos[0, 5, 0] = pos[1, 36, axes - 1] = -1                                  # padding
    qw, kw = weights(d, dtype, device, 3), weights(d, dtype, device, 4)
    shape = W.NormRopeShape(batch=B, n_tokens=T, n_q_heads=Hq, n_kv_heads=H, head_dim=d, dtype=dtype, inv_freq=inv, amplitude=amp, eps=eps, n_axes=axes,
                            axis_of_pair=axis if axes > 1 else None, interleaved=interleaved, q_strides=(T * n * d, d, n * d),
                            k_strides=(T * n * d, d, n * d), q_out_strides=(T * Hq * d, d, Hq * d), k_out_strides=(H * cap * d, cap * d, d))
    q_out = torch.full((B, T, Hq, d), 7.0, dtype=TYPES[dtype], device=device)
    cache = torch.full((B, H, cap, d), 7.0, dtype=TYPES[dtype], device=device)
    before = rows.clone()
    W.wkv_norm_rope(shape, pos, qw, kw, rows, q_out, rows[:, :, Hq:], cache)
    torch.cuda.synchronize()
    assert torch.equal(rows, before)
    for x, w, got in ((rows[:, :, :Hq], qw, q_out.transpose(1, 2)), (rows[:, :, Hq:Hq + H], kw, cache[:, :, :T])):
        want, size = expected(x.transpose(1, 2), w, pos, inv, axis, eps, amp, interleaved)
        padding = (pos.amin(-1) < 0)[:, None, :, None].expand_as(want)
        assert (got[padding] == 7.0).all(), "rows without a position are left alone"
        check(got[~padding], want[~padding], size[~padding], dtype)
    assert (cache[:, :, T:] == 7.0).all()


@pytest.mark.parametrize("B,T,Hq,H", [(1, 1, 1, 1), (64, 1, 32, 8), (3, 1, 28, 4), (1, 5, 0, 2), (2, 3, 9, 0), (1, 4099, 3, 1), (1, 9000, 1, 1), (2, 700, 64, 8)])
@pytest.mark.parametrize("q_norm,k_norm", [(True, True), (True, False), (False, True)])
def test_sizes_from_one_token_to_long_ones(device, B, T, Hq, H, q_norm, k_norm):
    d, dtype = 128, W.WKV_BF16
    inv, _ = W.wkv_rope_frequencies(d, 500000.0)
    g = torch.Generator(device=device).manual_seed(3)
    q = torch.randn((B, max(Hq, 1), T, d), device=device, generator=g).bfloat16()
    k = torch.randn((B, max(H, 1), T, d), device=device, generator=g).bfloat16()
    pos = (torch.arange(T, device=device, dtype=torch.int32) + 5).repeat(B, 1)[..., None].contiguous()
    qo, ko = torch.zeros_like(q), torch.zeros_like(k)
    qw, kw = (weights(d, dtype, device, 5) if q_norm else None), (weights(d, dtype, device, 6) if k_norm else None)
    shape = W.NormRopeShape(batch=B, n_tokens=T, n_q_heads=Hq, n_kv_heads=H, head_dim=d, dtype=dtype, inv_freq=inv)
    W.wkv_norm_rope(shape, pos, qw, kw, q if Hq else None, qo if Hq else None, k if H else None, ko if H else None)
    for x, w, got, heads in ((q, qw, qo, Hq), (k, kw, ko, H)):
        if heads:
            check(got, *expected(x, w, pos, inv, [0] * 64, 1e-6, 1.0, False), dtype)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("interleaved", [False, True])
def test_without_weights_it_is_the_rotation(device, dtype, interleaved):
    inv, amp = W.wkv_rope_frequencies(64, 10000.0, W.WKV_ROPE_PARTS, 4.0, 4096)
    x = torch.randn((2, 5, 300, 128), device=device, generator=torch.Generator(device=device).manual_seed(7)).to(TYPES[dtype])
    pos = torch.randint(0, 1 << 30, (2, 300), dtype=torch.int32, device=device, generator=torch.Generator(device=device).manual_seed(8))
    kw = dict(batch=2, n_tokens=300, n_q_heads=5, n_kv_heads=5, head_dim=128, dtype=dtype, inv_freq=inv, amplitude=amp, interleaved=interleaved)
    a, b, c, d = (torch.zeros_like(x) for _ in range(4))
    W.wkv_rope(W.RopeShape(**kw), pos, x, a, x, b)
    W.wkv_norm_rope(W.NormRopeShape(**kw), pos, None, None, x, c, x, d)
    # each is off by 2^-21 of a pair's magnitudes at most, and by one rounding to the type (of numbers up to those magnitudes): twice that apart
    half = torch.finfo(TYPES[dtype]).eps / 2
    size = expected(x, None, pos[..., None].clamp(max=1), inv, [0] * 32, 0.0, amp, interleaved)[1]
    for one, other in ((a, c), (b, d)):
        assert ((one.double() - other.double()).abs() <= 2 * size * (2.0 ** -21 + half) + 2.0 ** -24).all()
    # three axes with the same position on each are one, bit by bit
    W.wkv_norm_rope(W.NormRopeShape(n_axes=3, axis_of_pair=[i % 3 for i in range(32)], **kw), pos[..., None].repeat(1, 1, 3), None, None, x, a, x, b)
    assert torch.equal(a, c) and torch.equal(b, d)


def test_in_place_and_far_positions(device):
    inv, _ = W.wkv_rope_frequencies(64, 10000.0)
    x = torch.randn((2, 3, 11, 64), device=device, generator=torch.Generator(device=device).manual_seed(5))
    pos = torch.randint(2 ** 31 - 1000, 2 ** 31 - 1, (2, 11, 4), dtype=torch.int32, device=device)
    axis = [i % 4 for i in range(32)]
    w = weights(64, W.WKV_F32, device, 9)
    q, k = x.clone(), x.clone()
    W.wkv_norm_rope(W.NormRopeShape(batch=2, n_tokens=11, n_q_heads=3, n_kv_heads=3, head_dim=64, dtype=W.WKV_F32, inv_freq=inv, n_axes=4, axis_of_pair=axis),
                    pos, w, w, q, q, k, k)
    want, size = expected(x, w, pos, inv, axis, 1e-6, 1.0, False)
    # (64 bits leave 2^31 * 2^-53 of a radian in the oracle's angle: 2^-22)
    assert ((q.double() - want).abs() <= size * (2.0 ** -20 + 2.0 ** -21 + 2.0 ** -22) + want.abs() * 2.0 ** -24).all()
    assert torch.equal(q, k)


def test_sizes_of_rows_from_tiny_to_large(device):
    # a row's own size goes out of the result but for eps; rows of zeros stay zeros
    inv, _ = W.wkv_rope_frequencies(128, 10000.0)
    base = torch.randn((1, 1, 1, 128), device=device, generator=torch.Generator(device=device).manual_seed(10))
    x = torch.cat([base * f for f in (0.0, 1e-15, 1e-3, 1.0, 1e4, 1e15)], 2)
    pos = torch.full((1, 6, 1), 77, dtype=torch.int32, device=device)
    w = weights(128, W.WKV_F32, device, 11)
    y = torch.zeros_like(x)
    W.wkv_norm_rope(W.NormRopeShape(batch=1, n_tokens=6, n_q_heads=1, n_kv_heads=0, head_dim=128, dtype=W.WKV_F32, inv_freq=inv, eps=1e-6), pos, w, None, x, y, None, None)
    check(y, *expected(x, w, pos, inv, [0] * 64, 1e-6, 1.0, False), W.WKV_F32)
    assert not y[0, 0, 0].any()


def test_infinities_and_nan_stay_in_their_rows(device):
    inv, _ = W.wkv_rope_frequencies(64, 10000.0)
    x = torch.ones((1, 2, 3, 64), device=device)
    x[0, 0, 0, 3], x[0, 1, 2, 60] = math.nan, math.inf
    y = torch.zeros_like(x)
    W.wkv_norm_rope(W.NormRopeShape(batch=1, n_tokens=3, n_q_heads=2, n_kv_heads=0, head_dim=64, dtype=W.WKV_F32, inv_freq=inv),
                    torch.tensor([[[7], [8], [9]]], dtype=torch.int32, device=device), torch.ones(64, device=device), None, x, y, None, None)
    rows = torch.isfinite(y).all(-1)[0].tolist()
    assert rows == [[False, True, True], [True, True, False]]


def test_captured_and_replayed(device):
    inv, _ = W.wkv_rope_frequencies(128, 10000.0)
    shape = W.NormRopeShape(batch=4, n_tokens=1, n_q_heads=8, n_kv_heads=2, head_dim=128, dtype=W.WKV_BF16, inv_freq=inv)
    q, k = torch.randn((4, 8, 1, 128), device=device).bfloat16(), torch.randn((4, 2, 1, 128), device=device).bfloat16()
    qo, ko = torch.zeros_like(q), torch.zeros_like(k)
    qw, kw = weights(128, W.WKV_BF16, device, 12), weights(128, W.WKV_BF16, device, 13)
    pos = torch.tensor([[[1]], [[2]], [[3]], [[4]]], dtype=torch.int32, device=device)
    W.wkv_norm_rope(shape, pos, qw, kw, q, qo, k, ko)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        W.wkv_norm_rope(shape, pos, qw, kw, q, qo, k, ko)
    for step in range(3):
        pos += 1000 * step
        q.copy_(torch.randn_like(q.float()).bfloat16())
        graph.replay()
        torch.cuda.synchronize()
        check(qo, *expected(q, qw, pos, inv, [0] * 64, 1e-6, 1.0, False), W.WKV_BF16)
        check(ko, *expected(k, kw, pos, inv, [0] * 64, 1e-6, 1.0, False), W.WKV_BF16)


@pytest.mark.parametrize("dtype,d,interleaved,axes", [(W.WKV_BF16, 128, False, 1), (W.WKV_F16, 64, True, 3), (W.WKV_F32, 128, True, 1), (W.WKV_F32, 64, False, 2)])
def test_calls_past_the_memory_side_cache(device, dtype, d, interleaved, axes):
    # 300 MB of rows and more, in place, with padding among the tokens: the first tokens, the last ones and some between
    Hq, H = 7, 4
    T = 300 * 2 ** 20 // ((Hq + H) * d * TYPES[dtype].itemsize) + 3
    g = torch.Generator(device=device).manual_seed(20)
    rows = torch.randn((1, T, Hq + H, d), dtype=torch.float32, device=device, generator=g).to(TYPES[dtype])
    pos = torch.arange(T, dtype=torch.int32, device=device)[None, :, None] + torch.arange(axes, dtype=torch.int32, device=device)
    pos[0, 5::101, -1] = -1
    inv, _ = W.wkv_rope_frequencies(d, 10000.0)
    axis = [i % axes for i in range(d // 2)]
    qw, kw = weights(d, dtype, device, 21), weights(d, dtype, device, 22)
    at = torch.cat([torch.arange(0, 300), torch.arange(T // 2, T // 2 + 300), torch.arange(T - 300, T)]).to(device)
    before, where = rows[:, at].clone(), pos[:, at]
    n = (Hq + H) * d
    strides = (T * n, d, n)
    W.wkv_norm_rope(W.NormRopeShape(batch=1, n_tokens=T, n_q_heads=Hq, n_kv_heads=H, head_dim=d, dtype=dtype, inv_freq=inv, n_axes=axes, axis_of_pair=axis,
                                    interleaved=interleaved, q_strides=strides, q_out_strides=strides, k_strides=strides, k_out_strides=strides),
                    pos, qw, kw, rows, rows, rows[:, :, Hq:], rows[:, :, Hq:])
    padding = where[0, :, -1] < 0
    assert padding.any()
    assert torch.equal(rows[:, at][:, padding], before[:, padding])
    for part, w in ((slice(0, Hq), qw), (slice(Hq, Hq + H), kw)):
        want, size = expected(before[:, ~padding, part].transpose(1, 2), w, where[:, ~padding], inv, axis, 1e-6, 1.0, interleaved)
        check(rows[:, at][:, ~padding, part].transpose(1, 2), want, size, dtype)


def test_offsets_past_32_bits(device):
    # the second sequence 4.5 GiB behind the first, a second head 2.25 GiB behind the first
    d, T, half, far = 128, 3, 2 ** 30 + 2 ** 27, 2 ** 31 + 2 ** 28 + 1024
    buffer = torch.zeros(far + half + T * d, dtype=torch.bfloat16, device=device)
    x = buffer.as_strided((2, 2, T, d), (far, half, d, 1))
    x.copy_(torch.randn((2, 2, T, d), device=device, generator=torch.Generator(device=device).manual_seed(23)))
    before = x.clone()
    inv, _ = W.wkv_rope_frequencies(d, 10000.0)
    pos = torch.tensor([[[0], [7], [100]], [[3], [4], [5]]], dtype=torch.int32, device=device)
    w = weights(d, W.WKV_BF16, device, 24)
    W.wkv_norm_rope(W.NormRopeShape(batch=2, n_tokens=T, n_q_heads=0, n_kv_heads=2, head_dim=d, dtype=W.WKV_BF16, inv_freq=inv,
                                    k_strides=(far, half, d), k_out_strides=(far, half, d)), pos, None, w, None, None, x, x)
    check(x, *expected(before, w, pos, inv, [0] * 64, 1e-6, 1.0, False), W.WKV_BF16)
