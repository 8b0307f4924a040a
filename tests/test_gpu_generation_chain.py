"""The operators of generation together, as a program that serves long prompts uses them: normalised and turned queries and keys into the cache, the
window selection, its rows into 8 and 4 bits and generation over these; and over the plain compact caches trees of drafted tokens, of which a path is
kept, beside decode steps and an eviction.  Every stage is followed in 64 bits from the same inputs."""
import math

import pytest
import torch

import paper_2503_17922_amd as W
from tests import few_bits as F
from tests.test_gpu_norm_rope import check as check_norm_rope, expected as normed
from tests.test_gpu_tree import accepted, families, some_tree

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,fmt,Hq,H,d", [(W.WKV_BF16, W.WKV_CACHE_E4M3, 8, 2, 128), (W.WKV_F16, W.WKV_CACHE_E2M1, 7, 1, 64)])
def test_prompt_to_generation(device, dtype, fmt, Hq, H, d):
    t = torch.bfloat16 if dtype == W.WKV_BF16 else torch.float16
    half = torch.finfo(t).eps / 2
    B, lens, w, gamma, G, T = 2, [900, 611], 16, 2, Hq // H, 900
    win, k_win, room = 8, [24, 16], 60
    g = torch.Generator(device=device).manual_seed(21)
    inv, _ = W.wkv_rope_frequencies(d, 10000.0)
    n_heads = Hq + 2 * H
    pos = torch.full((B, T, 1), -1, dtype=torch.int32, device=device)
    for b, n in enumerate(lens):
        pos[b, :n, 0] = torch.arange(n, device=device)
    qw, kw = ((1 + 0.3 * torch.randn(d, device=device, generator=g)).to(t) for _ in range(2))
    shape = W.NormRopeShape(batch=B, n_tokens=T, n_q_heads=Hq, n_kv_heads=H, head_dim=d, dtype=dtype, inv_freq=inv,
                            q_strides=(T * n_heads * d, d, n_heads * d), k_strides=(T * n_heads * d, d, n_heads * d),
                            q_out_strides=(Hq * T * d, T * d, d), k_out_strides=(H * T * d, T * d, d))
    K, V, q_obs = [], [], None
    for layer in range(gamma):
        rows = (3 * torch.randn((B, T, n_heads, d), device=device, generator=g)).to(t)
        q, k = (torch.zeros((B, n, T, d), dtype=t, device=device) for n in (Hq, H))
        W.wkv_norm_rope(shape, pos, qw, kw, rows, q, rows[:, :, Hq:], k)
        for b, n in enumerate(lens):
            for x, weight, got in ((rows[b:b + 1, :n, :Hq], qw, q), (rows[b:b + 1, :n, Hq:Hq + H], kw, k)):
                check_norm_rope(got[b:b + 1, :, :n], *normed(x.transpose(1, 2), weight, pos[b:b + 1, :n], inv, [0] * (d // 2), 1e-6, 1.0, False), dtype)
        K.append(k); V.append(rows[:, :, Hq + H:].transpose(1, 2).contiguous())
        if layer == 0:
            q_obs = torch.stack([q[b, :, n - w:n] for b, n in enumerate(lens)]).contiguous()

    # ---- the selection, its rows into fewer bits and, for the trees, as they are
    p = W.Problem(n_q_heads=Hq, n_kv_heads=H, head_dim=d, w_obs=w, seq_len=lens, win=[win] * B, top_p=[win] * B, k_windows=k_win, dtype=dtype, max_seq_len=T)
    dims = W.wkv_get_dims(p)
    cap = dims.nkeep_max + room
    plain = W.Problem(n_q_heads=Hq, n_kv_heads=H, head_dim=d, w_obs=w, seq_len=lens, win=[win] * B, top_p=[win] * B, k_windows=k_win, dtype=dtype, max_seq_len=T,
                      out_strides=(H * cap * d, cap * d, d))
    ws = torch.empty(W.wkv_workspace_bytes(p), dtype=torch.uint8, device=device)
    scores, windows = torch.zeros((B, H, dims.t_stride), device=device), torch.zeros((B, H, dims.nw_max), device=device)
    win_idx, tok = torch.empty((B, H, dims.k_max), dtype=torch.int32, device=device), torch.empty((B, H, dims.nkeep_max), dtype=torch.int32, device=device)
    keep = torch.empty((B, H), dtype=torch.int32, device=device)
    W.wkv_score(p, q_obs, K[0], None, scores, ws)
    W.wkv_window_pool(p, scores, windows)
    W.wkv_topk_windows(p, windows, win_idx, tok, keep)
    row = d if fmt == W.WKV_CACHE_E4M3 else d // 2
    kq, vq = ([torch.zeros((B, H, cap, row), dtype=torch.uint8, device=device) for _ in range(gamma)] for _ in range(2))
    ks, vs = ([torch.zeros((B, H, cap, d // 32), dtype=torch.uint8, device=device) for _ in range(gamma)] for _ in range(2))
    put = W.QuantizedShape(batch=B, n_kv_heads=H, head_dim=d, dtype=dtype, format=fmt, capacity=cap, n_rows=dims.nkeep_max, row_capacity=T)
    W.wkv_cache_quantize(put, K, V, tok, keep, None, kq, ks, vq, vs)
    kc, vc = ([torch.zeros((B, H, cap, d), dtype=t, device=device) for _ in range(gamma)] for _ in range(2))
    W.wkv_gather_group(plain, K, V, tok, keep, kc, vc)
    for layer in range(gamma):
        for c, s, gathered in ((kq, ks, kc), (vq, vs, vc)):
            for b in range(B):
                for h in range(H):
                    n = int(keep[b, h])
                    codes, scales = F.encode(gathered[layer][b, h, :n], fmt)
                    assert torch.equal(c[layer][b, h, :n].cpu(), torch.from_numpy(codes)) and torch.equal(s[layer][b, h, :n].cpu(), torch.from_numpy(scales))
                    assert not c[layer][b, h, n:].any()

    # ---- generation over the caches in fewer bits; the layers share their counts
    n = keep.clone()
    kw_step = dict(batch=B, n_q_heads=Hq, n_kv_heads=H, head_dim=d, dtype=dtype, format=fmt, capacity=cap)
    last, before_last = W.QuantizedShape(**kw_step), W.QuantizedShape(flags=W.WKV_DECODE_KEEP_COUNT, **kw_step)
    ws_q = torch.empty(W.wkv_decode_quantized_workspace_bytes(last), dtype=torch.uint8, device=device)
    for step in range(4):
        for layer in range(gamma):
            q, k, v = (torch.randn((B, x, d), device=device, generator=g).to(t) for x in (Hq, H, H))
            out = torch.empty((B, Hq, d), device=device)
            was = n.clone()
            W.wkv_decode_step_quantized(last if layer == gamma - 1 else before_last, q, k, v, kq[layer], ks[layer], vq[layer], vs[layer], n, out, ws_q)
            for b in range(B):
                for h in range(H):
                    m = int(was[b, h])
                    assert int(n[b, h]) == m + (layer == gamma - 1)
                    for new, c, s in ((k, kq, ks), (v, vq, vs)):
                        codes, scales = F.encode(new[b, h][None], fmt)
                        assert torch.equal(c[layer][b, h, m].cpu(), torch.from_numpy(codes[0])) and torch.equal(s[layer][b, h, m].cpu(), torch.from_numpy(scales[0]))
                    k64, v64 = (F.decode_torch(c[layer][b, h, :m + 1], s[layer][b, h, :m + 1], fmt) for c, s in ((kq, ks), (vq, vs)))
                    share = torch.softmax(q[b, h * G:(h + 1) * G].double() @ k64.t() / math.sqrt(d), -1)
                    size = share @ v64.abs()
                    # (three parts of every number: what the step's own tests derive is below 2^-11 of the magnitudes at this size)
                    assert ((out[b, h * G:(h + 1) * G].double() - share @ v64).abs() <= 2.0 ** -11 * size).all()

    # ---- trees over the plain caches: drafted, checked, a path kept; a decode step in between, an eviction at the end
    n, at = keep.clone(), torch.tensor(lens, dtype=torch.int32, device=device)
    nodes = 10
    tree = W.TreeShape(batch=B, n_q_heads=Hq, n_kv_heads=H, head_dim=d, dtype=dtype, n_nodes=nodes, capacity=cap)
    decode = W.DecodeShape(batch=B, n_q_heads=Hq, n_kv_heads=H, head_dim=d, dtype=dtype, capacity=cap)
    keep_count = W.DecodeShape(batch=B, n_q_heads=Hq, n_kv_heads=H, head_dim=d, dtype=dtype, capacity=cap, flags=W.WKV_DECODE_KEEP_COUNT)
    ws_t = torch.empty(max(W.wkv_tree_workspace_bytes(tree), W.wkv_decode_workspace_bytes(decode)), dtype=torch.uint8, device=device)
    for turn in range(3):
        parents = [some_tree(nodes, 7 * turn + b) for b in range(B)]
        parent = torch.tensor(parents, dtype=torch.int32, device=device)
        depth = torch.tensor([[len(f) - 1 for f in families(x)] for x in parents], dtype=torch.int32, device=device)
        node_rope = W.NormRopeShape(batch=B, n_tokens=nodes, n_q_heads=Hq, n_kv_heads=H, head_dim=d, dtype=dtype, inv_freq=inv)
        new = [[], []]
        for layer in range(gamma):
            raw = [torch.randn((B, x, nodes, d), device=device, generator=g).to(t) for x in (Hq, H, H)]
            q, k, out = torch.zeros_like(raw[0]), torch.zeros_like(raw[1]), torch.zeros_like(raw[0])
            where = (at[:, None] + depth)[..., None].contiguous()
            W.wkv_norm_rope(node_rope, where, qw, kw, raw[0], q, raw[1], k)
            check_norm_rope(k, *normed(raw[1], kw, where, inv, [0] * (d // 2), 1e-6, 1.0, False), dtype)
            W.wkv_decode_tree(tree, q, k, raw[2], parent, kc[layer], vc[layer], n, out, ws_t)
            new[0].append(k); new[1].append(raw[2])
            for b in range(B):
                for h in range(H):
                    m = int(n[b, h])
                    for i, f in enumerate(families(parents[b])):
                        k64 = torch.cat([kc[layer][b, h, :m], k[b, h, f]]).double()
                        v64 = torch.cat([vc[layer][b, h, :m], raw[2][b, h, f]]).double()
                        share = torch.softmax(q[b, h * G:(h + 1) * G, i].double() @ k64.t() / math.sqrt(d), -1)
                        want, size = share @ v64, share @ v64.abs()
                        # a probability and the output rounded to the type, and as much as the tree's own tests derive for the rest (below 2^-9 at this size)
                        assert ((out[b, h * G:(h + 1) * G, i].double() - want).abs() <= want.abs() * half + size * (half + 2.0 ** -9)).all()
        paths = [f for f in (max(families(x), key=len) for x in parents)]
        path = torch.tensor([f + [-1] * (nodes - len(f)) for f in paths], dtype=torch.int32, device=device)
        accept = torch.tensor([turn, len(paths[1])], dtype=torch.int32, device=device)
        was = n.clone()
        W.wkv_tree_accept(tree, kc, vc, path, accept, n)
        assert torch.equal(n, was + accept.clamp(max=torch.tensor([len(f) for f in paths], device=device, dtype=torch.int32))[:, None])
        for layer in range(gamma):
            for c, x in ((kc, new[0][layer]), (vc, new[1][layer])):
                for b in range(B):
                    for h in range(H):
                        for i, node in enumerate(accepted(paths[b], int(accept[b]), nodes)):
                            assert torch.equal(c[layer][b, h, int(was[b, h]) + i], x[b, h, node])
        at += (n - was)[:, 0]
        for layer in range(gamma):
            q, k, v = (torch.randn((B, x, d), device=device, generator=g).to(t) for x in (Hq, H, H))
            out = torch.empty((B, Hq, d), device=device)
            W.wkv_decode_step(decode if layer == gamma - 1 else keep_count, q, k, v, kc[layer], vc[layer], n, out, ws_t)
            for b in range(B):
                for h in range(H):
                    m = int(n[b, h]) + (layer != gamma - 1)
                    share = torch.softmax(q[b, h * G:(h + 1) * G].double() @ kc[layer][b, h, :m].double().t() / math.sqrt(d), -1)
                    assert torch.allclose(out[b, h * G:(h + 1) * G].double(), share @ vc[layer][b, h, :m].double(), rtol=1e-3, atol=2e-5)
        at += 1
    assert torch.equal(n, keep + (at - torch.tensor(lens, dtype=torch.int32, device=device))[:, None])
    tok_of = torch.arange(cap, device=device, dtype=torch.int32).repeat(B, H, 1)
    weights = torch.rand((B, H, cap), device=device, generator=g)
    W.wkv_cache_evict(decode, kc, vc, weights, tok_of, n, keep, 4, torch.empty(W.wkv_evict_workspace_bytes(decode), dtype=torch.uint8, device=device))
    assert torch.equal(n, keep)
