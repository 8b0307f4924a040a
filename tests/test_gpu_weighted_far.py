"""The weighted decode step over caches whose rows lie past 32 bits, its outputs and weights against softmax(q K^T scale) in 64 bits: nothing there is rounded to 16 bits."""
import pytest
import torch

import paper_2503_17922_amd as W
from tests.test_gpu_decode_weighted import Caches
from tests.test_gpu_operator_extremes import FAR, give_memory_back, spread_out      # noqa: F401 (the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cap", [42, 1 << 28])          # a workgroup a cache, and ranges
@pytest.mark.parametrize("axis", ["head", "token"])
def test_outputs_and_weights(device, axis, cap):
    B, H, G, d, n = 3, 3, 2, 64, 40
    c = Caches(device, [n] * B, H * G, H, d, W.WKV_BF16, n + 2, seed=4)
    strides = dict(head=(H * FAR // 2, FAR // 2, d), token=((n + 2) * FAR // 64, d, FAR // 64))[axis]
    kc, vc = spread_out(c.kc, strides), spread_out(c.vc, strides)
    shape = W.DecodeShape(batch=B, n_q_heads=H * G, n_kv_heads=H, head_dim=d, dtype=W.WKV_BF16, capacity=cap, cache_strides=strides)
    weights, tok = torch.empty((B, H, cap), device=device), torch.empty((B, H, cap), dtype=torch.int32, device=device)
    weights[:, :, :n], tok[:, :, :n] = c.weights[:, :, :n], c.tok[:, :, :n]
    ws = torch.empty(W.wkv_decode_weighted_workspace_bytes(shape), dtype=torch.uint8, device=device)
    W.wkv_decode_step_weighted(shape, c.q, c.kn, c.vn, kc, vc, c.n, weights, tok, c.at, c.out, ws)
    c.kc[:, :, n], c.vc[:, :, n] = c.kn, c.vn
    assert torch.equal(kc, c.kc) and torch.equal(vc, c.vc) and (c.n == n + 1).all() and (tok[:, :, n] == c.at[:, None]).all()
    for b in range(B):
        for h in range(H):
            q, k, v = c.q[b, h * G:(h + 1) * G].double(), c.kc[b, h, :n + 1].double(), c.vc[b, h, :n + 1].double()
            p = torch.softmax(q @ k.t() * c.scale, -1)
            # a logit is off by (d + 4) 2^-24 scale |q| |k|, a probability by twice that and, with the sum of n terms and the exponents, (n + 16) 2^-24; sums of
            # products by as much again, the additions to a weight by half a step of the result each
            delta = (d + 4) * 2.0 ** -24 * c.scale * q.norm(dim=-1) * k.norm(dim=-1).max()
            loose = 2 * delta[:, None] + (n + 16) * 2.0 ** -24
            assert ((c.out[b, h * G:(h + 1) * G].double() - p @ v).abs() <= (p @ v.abs()) * (loose + (n + 16) * 2.0 ** -24)).all()
            want = c.weights[b, h, :n + 1].double()
            want[n] = 0.0
            want += p.sum(0)
            assert ((weights[b, h, :n + 1].double() - want).abs() <= (p * loose).sum(0) + (G + 1) * 2.0 ** -24 * want).all()
