"""The operators together, as a program that serves long prompts uses them: rotary positions into the cache, attention over the prompt, its
normalisers handed to the compression, generation with accumulated weights over the compact caches, eviction when they outgrow their budget.
Every stage is followed in 64 bits from the same inputs."""
import math

import pytest
import torch

import paper_2503_17922_amd as W
from tests.test_gpu_evict import expected
from tests.test_gpu_prefill_attention import check as check_attention
from tests.test_gpu_rope import check as check_rope, turned

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,Hq,H,d", [(W.WKV_BF16, 8, 2, 128), (W.WKV_F16, 7, 1, 64)])
def test_prompt_to_eviction(device, dtype, Hq, H, d):
    t = torch.bfloat16 if dtype == W.WKV_BF16 else torch.float16
    half = torch.finfo(t).eps / 2
    B, lens, w, gamma, G = 2, [1500, 901], 16, 2, Hq // H
    T, win, k_win, steps, recent = max(lens), 8, [40, 24], 12, 8
    g = torch.Generator(device=device).manual_seed(11)
    inv, amp = W.wkv_rope_frequencies(d, 10000.0, W.WKV_ROPE_WAVELENGTH, 2.0, 1024)
    n_heads = Hq + 2 * H
    pos = torch.full((B, T), -1, dtype=torch.int32, device=device)
    for b, n in enumerate(lens):
        pos[b, :n] = torch.arange(n, device=device)
    rope = W.RopeShape(batch=B, n_tokens=T, n_q_heads=Hq, n_kv_heads=H, head_dim=d, dtype=dtype, inv_freq=inv, amplitude=amp,
                       q_strides=(T * n_heads * d, d, n_heads * d), k_strides=(T * n_heads * d, d, n_heads * d),
                       q_out_strides=(Hq * T * d, T * d, d), k_out_strides=(H * T * d, T * d, d))
    att = W.AttentionShape(q_len=lens, n_q_heads=Hq, n_kv_heads=H, head_dim=d, dtype=dtype, lse_rows=w,
                           q_strides=(Hq * T * d, T * d, d), kv_strides=(H * T * d, T * d, d))
    ws_att = torch.empty(W.wkv_attention_workspace_bytes(att), dtype=torch.uint8, device=device)

    # ---- the prompt, layer by layer
    K, V, lse, q_obs = [], [], None, None
    for layer in range(gamma):
        rows = torch.randn((B, T, n_heads, d), device=device, generator=g).to(t)
        q, out, k = (torch.zeros((B, n, T, d), dtype=t, device=device) for n in (Hq, Hq, H))
        v = rows[:, :, Hq + H:].transpose(1, 2).contiguous()
        W.wkv_rope(rope, pos, rows, q, rows[:, :, Hq:], k)
        lse_layer = torch.empty((B, Hq, w), device=device)
        W.wkv_prefill_attention(att, q, k, v, out, lse_layer, ws_att)
        for b, n in enumerate(lens):
            for x, got in ((rows[b:b + 1, :n, :Hq], q), (rows[b:b + 1, :n, Hq:Hq + H], k)):
                check_rope(got[b:b + 1, :, :n], *turned(x.transpose(1, 2), pos[b:b + 1, :n], inv, amp, False), dtype)
            check_attention(out[b, :, :n], lse_layer[b], q[b, :, :n], k[b, :, :n], v[b, :, :n], d ** -0.5, dtype)
        K.append(k); V.append(v)
        if layer == 0:
            lse, q_obs = lse_layer, torch.stack([q[b, :, n - w:n] for b, n in enumerate(lens)]).contiguous()

    # ---- compression, with the normalisers of the attention
    budget = max(k * win + w for k in k_win)
    cap = budget + 5
    p = W.Problem(n_q_heads=Hq, n_kv_heads=H, head_dim=d, w_obs=w, seq_len=lens, win=[win] * B, top_p=[win] * B, k_windows=k_win, dtype=dtype,
                  out_strides=(H * cap * d, cap * d, d))
    dims = W.wkv_get_dims(p)
    assert dims.nkeep_max == budget
    kc, vc = ([torch.zeros((B, H, cap, d), dtype=t, device=device) for _ in range(gamma)] for _ in range(2))
    win_idx = torch.empty((1, B, H, dims.k_max), dtype=torch.int32, device=device)
    tok_k, n = torch.empty((1, B, H, budget), dtype=torch.int32, device=device), torch.empty((1, B, H), dtype=torch.int32, device=device)
    ws = torch.empty(W.wkv_workspace_bytes(p), dtype=torch.uint8, device=device)
    W.wkv_compress_groups(p, 1, gamma, [q_obs], [lse], K, V, kc, vc, win_idx, tok_k, n, ws)
    scores = torch.zeros((B, H, dims.t_stride), device=device)
    W.wkv_score(p, q_obs, K[0], lse, scores, ws)
    n, tok = n[0], torch.zeros((B, H, cap), dtype=torch.int32, device=device)
    tok[:, :, :budget] = tok_k[0]
    weights = torch.zeros((B, H, cap), device=device)
    for b in range(B):
        # token scores in 64 bits: what every retained row has received from the observation rows
        last = lens[b] - w
        for h in range(H):
            logits = q_obs[b, h * G:(h + 1) * G].double().reshape(-1, d) @ K[0][b, h, :lens[b]].double().t() / math.sqrt(d)
            hidden = torch.arange(lens[b], device=device)[None] > (torch.arange(w, device=device) + last).repeat(G)[:, None]
            t64 = torch.softmax(logits.masked_fill(hidden, -math.inf), -1).sum(0)
            assert torch.allclose(scores[b, h, :last].double(), t64[:last], rtol=2e-3, atol=1e-9)
            kept = tok[b, h, :int(n[b, h])].long()
            weights[b, h, :len(kept)] = torch.where(kept < last, scores[b, h, kept.clamp(max=last - 1)], torch.zeros((), device=device))

    # ---- generation; the cache of the first layer decides for both
    decode = W.DecodeShape(batch=B, n_q_heads=Hq, n_kv_heads=H, head_dim=d, dtype=dtype, capacity=cap)
    keep_count = W.DecodeShape(batch=B, n_q_heads=Hq, n_kv_heads=H, head_dim=d, dtype=dtype, capacity=cap, flags=W.WKV_DECODE_KEEP_COUNT)
    ws_w = torch.empty(W.wkv_decode_weighted_workspace_bytes(keep_count), dtype=torch.uint8, device=device)
    ws_e = torch.empty(W.wkv_evict_workspace_bytes(decode), dtype=torch.uint8, device=device)
    step_rope = W.RopeShape(batch=B, n_tokens=1, n_q_heads=Hq, n_kv_heads=H, head_dim=d, dtype=dtype, inv_freq=inv, amplitude=amp)
    keep = n.clone()
    at = torch.tensor(lens, dtype=torch.int32, device=device)
    evictions = 0
    for step in range(steps):
        for layer in range(gamma):
            raw = [torch.randn((B, x, 1, d), device=device, generator=g).to(t) for x in (Hq, H, H)]
            q, k = torch.zeros_like(raw[0]), torch.zeros_like(raw[1])
            W.wkv_rope(step_rope, at[:, None].contiguous(), raw[0], q, raw[1], k)
            check_rope(k, *turned(raw[1], at[:, None], inv, amp, False), dtype)
            out = torch.empty((B, Hq, d), device=device)
            before_n, before_w = n.clone(), weights.clone()
            if layer == 0:
                W.wkv_decode_step_weighted(keep_count, q, k, raw[2], kc[0], vc[0], n, weights, tok, at, out, ws_w)
            else:
                W.wkv_decode_step(decode, q, k, raw[2], kc[1], vc[1], n, out, ws_w)
            for b in range(B):
                for h in range(H):
                    m = int(before_n[b, h])
                    assert int(n[b, h]) == m + layer
                    assert torch.equal(kc[layer][b, h, m], k[b, h, 0]) and torch.equal(vc[layer][b, h, m], raw[2][b, h, 0])
                    share = torch.softmax(q[b, h * G:(h + 1) * G, 0].double() @ kc[layer][b, h, :m + 1].double().t() / math.sqrt(d), -1)
                    assert torch.allclose(out[b, h * G:(h + 1) * G].double(), share @ vc[layer][b, h, :m + 1].double(), rtol=1e-3, atol=2e-5)
                    if layer == 0:
                        want = before_w[b, h, :m + 1].double()
                        want[m] = 0
                        assert torch.allclose(weights[b, h, :m + 1].double(), want + share.sum(0), rtol=1e-4, atol=1e-7)
                        assert int(tok[b, h, m]) == int(at[b])
        if int(n.max()) >= cap - 1 or step == 3:
            evictions += 1
            was = [x.clone() for x in kc + vc + [weights, tok]]
            rows = n.clone()
            W.wkv_cache_evict(decode, kc, vc, weights, tok, n, keep, recent, ws_e)
            assert torch.equal(n, keep)
            for b in range(B):
                for h in range(H):
                    source = expected(was[-2][b, h].cpu().numpy(), was[-1][b, h].cpu().numpy(), int(rows[b, h]), int(keep[b, h]), recent)
                    ii = torch.from_numpy(source).to(device)
                    for x, y in zip(kc + vc + [weights, tok], was):
                        assert torch.equal(x[b, h, :len(ii)], y[b, h][ii])
                    # the last tokens are there, whatever their weight
                    newest = set(range(int(at[b]) - recent + 1, int(at[b]) + 1))
                    assert newest <= set(tok[b, h, :len(ii)].tolist())
        at += 1
    assert evictions >= 3
