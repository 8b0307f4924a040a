"""The parts that wkv_decode_step_quantized cuts queries and probabilities into, at inputs where each of them shows: keys and values of a single channel, so that a logit is one
product and an output one probability, with bounds of a few steps of fp32.  That results without the last part are outside of the bounds is checked on the CPU."""
import math

import pytest
import torch

import paper_2503_17922_amd as W

TYPES = {W.WKV_F32: torch.float32, W.WKV_BF16: torch.bfloat16, W.WKV_F16: torch.float16}
LIVE = 24                                                      # rows that weigh anything


def inputs(d, G, dtype, n, at, large, seed):
    """Plain rows of n + 1 tokens (the last is the new one): rows at .. at + LIVE - 2 and the new one are unit vectors, channel i the i-th of them; all others are the last channel's,
    whose logits are far below.  large: logits of about 100, of a query in fp32 the part after the
    first nearly half a step of that, and the third nearly half a step of the second; otherwise logits up to 3."""
    g = torch.Generator().manual_seed(seed)
    unit = torch.zeros(n + 1, d)
    live = list(range(at, at + LIVE - 1)) + [n]
    unit[:, d - 1] = 1.0
    for i, r in enumerate(live):
        unit[r] = 0.0
        unit[r, i] = 1.0
    if large:
        q = 100.0 + torch.rand(G, d, generator=g) * 6 - 3
        if dtype == W.WKV_F32:
            low = torch.where(torch.rand(G, d, generator=g) < 0.5, 0x7f3f, 0x80c1)
            q = ((q.view(torch.int32) & ~0xffff) | low.to(torch.int32)).view(torch.float32)
        q[:, d - 1] = -100.0
    else:
        q = torch.rand(G, d, generator=g) * 6 - 3
        q[:, d - 1] = -100.0
    return q.to(TYPES[dtype]), unit, live


def bounds(q, unit, live):
    """Outputs in 64 bits and how far they may be off, with logit scale 1 and rows held exactly.
    A logit is exact: one product of each part with a power of two.  Its product with log2(e) and the difference to a reference are rounded, 2^-24 each of numbers up to
    1.4427 |s| and 2.9 max |s - s'| + 8 (the reference lags by up to 2^8): the probability is off by ln 2 of that, and by 2^-23 of the exponential.  The rescalings of waves and ranges
    are two exponentials more, of differences as large.  A sum of LIVE probabilities adds LIVE steps, its three parts' products and sums with zeros 4, the division and the last
    products 4.  Numerator and denominator are off by one probability's error each."""
    s = q.double() @ unit.double().t()
    want = torch.softmax(s, -1)[:, live]
    top = s[:, live]
    spread = float(top.max() - top.min())
    size = float(top.abs().max())
    one = math.log(2) * (1.4427 * size + 1.4427 * spread + 8) + 2 + 2 * (math.log(2) * (1.4427 * spread + 8) + 2)
    return want, want * (2 * one + LIVE + 8) * 2.0 ** -24


def bf16(x):
    return x.to(torch.bfloat16).to(torch.float32)


@pytest.mark.parametrize("d", [64, 128])
def test_the_bounds_see_a_missing_part(d):
    q, unit, live = inputs(d, 8, W.WKV_F32, 31, 3, True, 1)
    want, tol = bounds(q, unit, live)
    two = bf16(q) + bf16(q - bf16(q))                          # queries without their third part
    short = torch.softmax(two.double() @ unit.double().t(), -1)[:, live]
    assert (short - want).abs().div(tol).max() > 10
    whole = two + bf16(q - two)
    assert torch.equal(whole, q)
    q, unit, live = inputs(d, 8, W.WKV_F16, 31, 3, True, 2)
    want, tol = bounds(q, unit, live)
    short = torch.softmax(bf16(q.float()).double() @ unit.double().t(), -1)[:, live]
    assert (short - want).abs().div(tol).max() > 100
    q, unit, live = inputs(d, 8, W.WKV_BF16, 31, 3, False, 3)
    want, tol = bounds(q, unit, live)
    s = (q.float() @ unit.t())
    p = torch.exp2((s - s.amax(-1, keepdim=True)) * 1.4426950408889634)
    cut = (p.view(torch.int32) & ~0xff).view(torch.float32)    # probabilities without their last eight bits
    short = (cut.double() / p.double().sum(-1, keepdim=True))[:, live]
    assert (short - want).abs().div(tol).max() > 1.5
    assert ((p.double() / p.double().sum(-1, keepdim=True))[:, live] - want).abs().le(tol).all()


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", [W.WKV_CACHE_E4M3, W.WKV_CACHE_E2M1])
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [1, 3, 4, 5, 8])
def test_every_part_counts(device, fmt, dtype, d, G):
    for large in (True, False):
        for n, at in ((31, 3), (32, 0), (120, 40), (130, 101), (400, 250)):
            q, unit, live = inputs(d, G, dtype, n, at, large, 10 * n + G)
            want, tol = bounds(q, unit, live)
            cap = n + 3
            row = d if fmt == W.WKV_CACHE_E4M3 else d // 2
            codes = [torch.zeros((1, 1, cap, row), dtype=torch.uint8, device=device) for _ in range(2)]
            scales = [torch.zeros((1, 1, cap, d // 32), dtype=torch.uint8, device=device) for _ in range(2)]
            plain = unit.to(device)[None, None, :n].contiguous()
            W.wkv_cache_quantize(W.QuantizedShape(batch=1, n_kv_heads=1, head_dim=d, dtype=W.WKV_F32, format=fmt, capacity=cap, n_rows=n), [plain], [plain], None, None, None,
                                 [codes[0]], [scales[0]], [codes[1]], [scales[1]])
            sh = W.QuantizedShape(batch=1, n_q_heads=G, n_kv_heads=1, head_dim=d, dtype=dtype, format=fmt, capacity=cap, scale=1.0)
            new = unit[n].to(TYPES[dtype]).to(device).view(1, 1, d)
            out = torch.zeros((1, G, d), device=device)
            W.wkv_decode_step_quantized(sh, q.to(device)[None].contiguous(), new, new, codes[0], scales[0], codes[1], scales[1], torch.tensor([[n]], dtype=torch.int32, device=device), out,
                                        torch.empty(W.wkv_decode_quantized_workspace_bytes(sh), dtype=torch.uint8, device=device))
            err = (out[0, :, :LIVE].double().cpu() - want).abs()
            assert (err <= tol).all(), f"n {n} large {large}: worst {float((err / tol).max())} of the bound"
