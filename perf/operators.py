"""The operators around the compression of a KV cache and the calls they are measured by: rotary positions, attention
over a prompt, the decode step that accumulates attention weights, and eviction by them.

A case is a dict of plain values.  ``kind`` names the operator:

rope      ``wkv_rope``: queries and keys of ``lens`` tokens a sequence (padded to the longest), read from the rows of one
          fused projection [batch, token, (q | k | v) heads, channel], keys written into a cache [batch, head, row, channel].
          ``scaling``: none, linear, base, parts or wavelength, by ``factor``.
prefill   ``wkv_prefill_attention``: ``lens`` new tokens a sequence after ``past`` earlier ones.  ``layout``: "packed" (the
          sequences one after the other, token-major) or "padded" ([batch, head, row, channel]).  ``lse_rows``: normalisers
          of that many last rows a sequence, as the score call takes them.
weighted  ``wkv_decode_step_weighted``: one token over caches of ``rows`` rows (one number a sequence).
evict     ``wkv_cache_evict``: caches of ``rows`` rows cut to ``keep`` in ``layers`` layers, the last ``recent`` tokens protected.

Where ``own`` is false, ``run`` computes an operator from elementary torch operations in 32 bits (angles in 64).
"""
import math

import torch

own = False

_TORCH = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_ROOM = 256              # rows a cache has for tokens to come


def _wkv():
    import paper_2503_17922_amd as W
    return W


def _dtype(W, name):
    return {"bf16": W.WKV_BF16, "f16": W.WKV_F16, "f32": W.WKV_F32}[name]


def _ints(text):
    return [int(x) for x in str(text).split()]


def _text(xs):
    return " ".join(str(x) for x in xs)


def _rope(name, lens, **kw):
    c = dict(name=name, kind="rope", dtype="bf16", q_heads=32, kv_heads=8, head_dim=128, rotary=128, interleaved=False,
             lens=_text(lens), first=0, theta=500000.0, scaling="none", factor=1.0, original=8192)
    c.update(kw)
    return c


def _prefill(name, lens, **kw):
    c = dict(name=name, kind="prefill", dtype="bf16", q_heads=32, kv_heads=8, head_dim=128, lens=_text(lens),
             past=_text([0] * len(lens)), layout="padded", lse_rows=32)
    c.update(kw)
    return c


def _weighted(name, rows, **kw):
    c = dict(name=name, kind="weighted", dtype="bf16", q_heads=32, kv_heads=8, head_dim=128, rows=_text(rows))
    c.update(kw)
    return c


def _evict(name, rows, **kw):
    c = dict(name=name, kind="evict", dtype="bf16", kv_heads=8, head_dim=128, layers=4, rows=_text(rows), keep=4096, recent=32)
    c.update(kw)
    return c


def listed():
    return [
        # the new token of each of 64 sequences that generate together: latency
        _rope("rope_step_64", [1] * 64, first=4096),
        # the prompt of the 32K benchmark, frequencies scaled by wavelength for a context longer than trained
        _rope("rope_prompt_32k", [32768], scaling="wavelength", factor=8.0),
        # a padded batch of odd lengths, interleaved pairs in half of a head's channels, scaled by parts, half precision
        _rope("rope_ragged_f16", [9973, 2051, 5003], dtype="f16", q_heads=28, kv_heads=4, rotary=64, interleaved=True,
              scaling="parts", factor=4.0, theta=10000.0, original=4096),
        # a short prompt of a small model in fp32: launches and the start of a workgroup are all there is
        _prefill("prefill_tiny_f32", [512], dtype="f32", q_heads=4, kv_heads=2, head_dim=64, lse_rows=8),
        # an ordinary prompt of a LLaMA-3-8B shaped model
        _prefill("prefill_4k", [4096]),
        # the prompt of the 32K benchmark: the largest call
        _prefill("prefill_32k", [32768]),
        # prompts of very different lengths one after the other in one tensor, seven query heads to a KV head, half precision
        _prefill("prefill_packed_f16", [9973, 2051, 1, 5003, 377], dtype="f16", q_heads=28, kv_heads=4, layout="packed", lse_rows=0),
        # the last piece of a 32K prompt that is taken in pieces: few new rows over a long cache
        _prefill("prefill_piece", [200], past="32568"),
        # one user's token over a compact cache: latency
        _weighted("weighted_1", [4128]),
        # generation at full batch
        _weighted("weighted_64", [4128] * 64),
        # one row too many in one user's cache: latency
        _evict("evict_1", [4097]),
        # a batch whose caches ran past their budget by different amounts, all layers of a group
        _evict("evict_mixed", [5120, 4096, 4481, 7777, 4999, 8192, 4100, 6003]),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_HEADS = [(32, 8), (32, 8), (64, 8), (28, 4), (12, 2), (32, 32)]


def draw(rng):
    kind = rng.choice(["rope", "prefill", "prefill", "weighted", "evict"])
    q, kv = rng.choice(_HEADS)
    d = rng.choice([64, 128, 128])
    c = dict(kind=kind, dtype=rng.choice(["bf16"] * 5 + ["f16"] * 3 + ["f32"]), q_heads=q, kv_heads=kv, head_dim=d)
    if kind == "rope":
        batch = _log(rng, 1, 64)
        longest = _log(rng, 1, 32768 // batch)
        rotary = rng.choice([d, d, d // 2, d // 4])
        scaling = rng.choice(["none", "linear", "base", "parts", "wavelength"])
        c.update(rotary=rotary, interleaved=rng.random() < 0.4, first=rng.choice([0, 0, _log(rng, 1, 100000)]),
                 lens=_text([longest] + [_log(rng, max(1, longest // 8), longest) for _ in range(batch - 1)]),
                 theta=rng.choice([10000.0, 500000.0, 1000000.0]), scaling=scaling,
                 factor=1.0 if scaling == "none" else rng.choice([2.0, 4.0, 8.0]), original=rng.choice([4096, 8192]))
    elif kind == "prefill":
        batch = _log(rng, 1, 16)
        longest = _log(rng, 16, 16384 if c["dtype"] != "f32" else 4096) // (1 + batch // 4) + 1
        lens = [longest] + [_log(rng, max(1, longest // 16), longest) for _ in range(batch - 1)]
        past = [_log(rng, 1, 16384 if c["dtype"] != "f32" else 4096) if rng.random() < 0.7 else 0 for _ in lens] if rng.random() < 0.3 else [0] * batch
        if max(past) > 0:
            lens = [min(n, 1024) for n in lens]
        c.update(lens=_text(lens), past=_text(past), layout=rng.choice(["packed", "padded"]), lse_rows=rng.choice([0, 8, 32]))
    elif kind == "weighted":
        batch = _log(rng, 1, 48)
        longest = _log(rng, 64, 16384) // (1 + batch // 8) + 1
        c.update(rows=_text([longest] + [_log(rng, max(1, longest // 8), longest) for _ in range(batch - 1)]))
    else:
        batch = _log(rng, 1, 32)
        keep = _log(rng, 100, 8192)
        layers = rng.choice([1, 2, 4])
        c.update(layers=layers, keep=keep, recent=rng.choice([0, 8, 32]),
                 rows=_text(rng.choice([keep + 1, _log(rng, max(keep // 2, 1), 2 * keep)]) for _ in range(batch)))
        del c["q_heads"]
    return c


# ---- inputs ---------------------------------------------------------------------------------------------------------

def _frequencies(case):
    """Inverse frequencies (64 bits) and the amplitude of the rotation."""
    r, theta, s, original = case["rotary"], case["theta"], case["factor"], case["original"]
    plain = [theta ** (-2.0 * i / r) for i in range(r // 2)]
    kind = case["scaling"]
    if kind == "linear":
        return [f / s for f in plain], 1.0
    if kind == "base":
        wider = theta * s ** (r / (r - 2.0))
        return [wider ** (-2.0 * i / r) for i in range(r // 2)], 1.0
    if kind == "parts":
        # a channel that makes `fast` turns or more within the original context keeps its frequency, one that
        # makes `slow` turns or fewer is slowed by the whole factor, linearly by channel number in between
        fast, slow = 32.0, 1.0
        at = [r * math.log(original / (n * 2.0 * math.pi)) / (2.0 * math.log(theta)) for n in (fast, slow)]
        lo, hi = max(math.floor(at[0]), 0), min(math.ceil(at[1]), r - 1)
        out = []
        for i, f in enumerate(plain):
            ramp = min(max((i - lo) / (hi - lo if hi != lo else 0.001), 0.0), 1.0)
            out.append(f * (1.0 - ramp) + f / s * ramp)
        return out, 0.1 * math.log(s) + 1.0
    if kind == "wavelength":
        low, high = 1.0, 4.0
        out = []
        for f in plain:
            turns = original * f / (2.0 * math.pi)
            mix = min(max((turns - low) / (high - low), 0.0), 1.0)
            out.append(f * mix + f / s * (1.0 - mix))
        return out, 1.0
    return plain, 1.0


def _normal(g, shape, dtype, scale=1.0):
    return (torch.randn(shape, device="cuda", dtype=torch.float32, generator=g) * scale).to(_TORCH[dtype])


def _starts(lens):
    out = [0]
    for n in lens:
        out.append(out[-1] + n)
    return out


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    d, kv, dt = case["head_dim"], case["kv_heads"], case["dtype"]
    kind = case["kind"]
    st = dict(case=case)
    if kind == "rope":
        lens, q = _ints(case["lens"]), case["q_heads"]
        B, T = len(lens), max(lens)
        rows = _normal(g, (B, T, q + 2 * kv, d), dt)
        pos = torch.full((B, T), -1, dtype=torch.int32, device="cuda")       # padding
        for b, n in enumerate(lens):
            pos[b, :n] = torch.arange(n, device="cuda", dtype=torch.int32) + case["first"] + 7 * b
        inv, amp = _frequencies(case)
        st.update(q=rows[:, :, :q], k=rows[:, :, q:q + kv], pos=pos,
                  inv=torch.tensor(inv, dtype=torch.float64, device="cuda"), amp=amp, inv_host=inv,
                  q_out=torch.zeros((B, T, q, d), dtype=_TORCH[dt], device="cuda"),
                  k_out=torch.zeros((B, kv, T + _ROOM, d), dtype=_TORCH[dt], device="cuda"))
        if own:
            W = _wkv()
            kinds = dict(none=W.WKV_ROPE_PLAIN, linear=W.WKV_ROPE_LINEAR, base=W.WKV_ROPE_BASE, parts=W.WKV_ROPE_PARTS,
                         wavelength=W.WKV_ROPE_WAVELENGTH)
            freq, amplitude = W.wkv_rope_frequencies(case["rotary"], case["theta"], kinds[case["scaling"]], case["factor"],
                                                     case["original"])
            h = q + 2 * kv
            st["shape"] = W.RopeShape(batch=B, n_tokens=T, n_q_heads=q, n_kv_heads=kv, head_dim=d, dtype=_dtype(W, dt),
                                      inv_freq=freq, amplitude=amplitude, interleaved=case["interleaved"],
                                      q_strides=(T * h * d, d, h * d), k_strides=(T * h * d, d, h * d),
                                      q_out_strides=(T * q * d, d, q * d), k_out_strides=(kv * (T + _ROOM) * d, (T + _ROOM) * d, d))
    elif kind == "prefill":
        lens, past, q = _ints(case["lens"]), _ints(case["past"]), case["q_heads"]
        total = [n + p for n, p in zip(lens, past)]
        B, packed = len(lens), case["layout"] == "packed"
        if packed:
            shape_q, shape_k = (sum(lens), q, d), (sum(total), kv, d)
        else:
            shape_q, shape_k = (B, q, max(lens), d), (B, kv, max(total), d)
        # logits of a standard deviation of 1.5, a few rows of which single keys dominate
        st.update(q=_normal(g, shape_q, dt, 1.5), k=_normal(g, shape_k, dt), v=_normal(g, shape_k, dt))
        st["out"] = torch.zeros(shape_q, dtype=_TORCH[dt], device="cuda")
        st["lse"] = torch.zeros((B, q, case["lse_rows"]), dtype=torch.float32, device="cuda") if case["lse_rows"] else None
        if own:
            W = _wkv()
            kw = dict(q_len=lens, k_len=total, n_q_heads=q, n_kv_heads=kv, head_dim=d, dtype=_dtype(W, dt), lse_rows=case["lse_rows"])
            if packed:
                kw.update(q_strides=(0, d, q * d), out_strides=(0, d, q * d), kv_strides=(0, d, kv * d),
                          q_start=_starts(lens)[:-1], k_start=_starts(total)[:-1])
            st["shape"] = W.AttentionShape(**kw)
            st["ws"] = torch.empty(W.wkv_attention_workspace_bytes(st["shape"]), dtype=torch.uint8, device="cuda")
    elif kind == "weighted":
        rows, q = _ints(case["rows"]), case["q_heads"]
        B, cap = len(rows), max(rows) + _ROOM
        st.update(q=_normal(g, (B, q, d), dt, 1.5), kn=_normal(g, (B, kv, d), dt), vn=_normal(g, (B, kv, d), dt),
                  kc=_normal(g, (B, kv, cap, d), dt), vc=_normal(g, (B, kv, cap, d), dt),
                  n=torch.tensor(rows, dtype=torch.int32, device="cuda")[:, None].repeat(1, kv),
                  start=torch.rand((B, kv, cap), device="cuda", generator=g) * 4.0,
                  weights=torch.empty((B, kv, cap), device="cuda"),
                  tok=torch.arange(cap, device="cuda", dtype=torch.int32).repeat(B, kv, 1),
                  at=torch.tensor([8 * n for n in rows], dtype=torch.int32, device="cuda"),
                  out=torch.empty((B, q, d), device="cuda"), rows=rows)
        if own:
            W = _wkv()
            st["shape"] = W.DecodeShape(batch=B, n_q_heads=q, n_kv_heads=kv, head_dim=d, dtype=_dtype(W, dt), capacity=cap,
                                        flags=W.WKV_DECODE_KEEP_COUNT)
            st["ws"] = torch.empty(W.wkv_decode_weighted_workspace_bytes(st["shape"]), dtype=torch.uint8, device="cuda")
    else:
        rows = _ints(case["rows"])
        B, cap = len(rows), max(rows) + _ROOM
        # a row's weight: most rows get little, a few much
        weights = torch.rand((B, kv, cap), device="cuda", generator=g) ** 8 * 4.0
        step = torch.randint(1, 8, (B, kv, cap), device="cuda", generator=g)
        tok = torch.cumsum(step, -1).to(torch.int32)
        n = torch.tensor(rows, dtype=torch.int32, device="cuda")[:, None].repeat(1, kv)
        # what an eviction changes besides the caches, in one buffer, and its first state: weights, positions, counts
        cells = B * kv * cap
        first = torch.cat([weights.flatten().view(torch.int32), tok.flatten(), n.flatten()])
        state = first.clone()
        st.update(first=first, state=state, weights=state[:cells].view(torch.float32).view(B, kv, cap),
                  tok=state[cells:2 * cells].view(B, kv, cap), n=state[2 * cells:].view(B, kv),
                  keep=torch.full((B, kv), case["keep"], dtype=torch.int32, device="cuda"),
                  kc=[_normal(g, (B, kv, cap, d), dt) for _ in range(case["layers"])],
                  vc=[_normal(g, (B, kv, cap, d), dt) for _ in range(case["layers"])], rows=rows)
        if own:
            W = _wkv()
            st["shape"] = W.DecodeShape(batch=B, n_q_heads=kv, n_kv_heads=kv, head_dim=d, dtype=_dtype(W, dt), capacity=cap)
            st["ws"] = torch.empty(W.wkv_evict_workspace_bytes(st["shape"]), dtype=torch.uint8, device="cuda")
    return st


# ---- one pass -------------------------------------------------------------------------------------------------------

def _turn(x, cos, sin, case):
    """Pairs of the first ``rotary`` channels of x [B, T, H, d] turned by angles given as cos and sin [B, T, 1, rotary / 2]."""
    r = case["rotary"]
    y = x.float()
    if case["interleaved"]:
        a, b = y[..., 0:r:2], y[..., 1:r:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = y[..., :r // 2], y[..., r // 2:r]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turned, y[..., r:]], -1).to(x.dtype)


def _plain_rope(st):
    c = st["case"]
    T = st["pos"].shape[1]
    angle = st["pos"].double()[:, :, None, None] * st["inv"]
    cos, sin = (torch.cos(angle) * st["amp"]).float(), (torch.sin(angle) * st["amp"]).float()
    valid = (st["pos"] >= 0)[:, :, None, None]
    st["q_out"].copy_(torch.where(valid, _turn(st["q"], cos, sin, c), st["q_out"]))
    k_rows = st["k_out"][:, :, :T].transpose(1, 2)
    k_rows.copy_(torch.where(valid, _turn(st["k"], cos, sin, c), k_rows))


def _rows_of(st, b, lens, total, packed):
    """Views of sequence b: queries and outputs [head, row, channel], keys and values likewise."""
    if packed:
        q0, k0 = sum(lens[:b]), sum(total[:b])
        pick = lambda t, at, n: t[at:at + n].transpose(0, 1)
        return pick(st["q"], q0, lens[b]), pick(st["out"], q0, lens[b]), pick(st["k"], k0, total[b]), pick(st["v"], k0, total[b])
    return st["q"][b, :, :lens[b]], st["out"][b, :, :lens[b]], st["k"][b, :, :total[b]], st["v"][b, :, :total[b]]


def _plain_prefill(st):
    c = st["case"]
    lens, past = _ints(c["lens"]), _ints(c["past"])
    total = [n + p for n, p in zip(lens, past)]
    G, scale = c["q_heads"] // c["kv_heads"], c["head_dim"] ** -0.5
    for b, n in enumerate(lens):
        q, out, k, v = _rows_of(st, b, lens, total, c["layout"] == "packed")
        for h in range(c["kv_heads"]):
            kf, vf = k[h].float(), v[h].float()
            for r0 in range(0, n, 4096):
                r1 = min(r0 + 4096, n)
                seen = past[b] + r1
                hidden = torch.arange(seen, device="cuda")[None, :] > (torch.arange(r0, r1, device="cuda") + past[b])[:, None]
                for head in range(h * G, (h + 1) * G):
                    s = (q[head, r0:r1].float() @ kf[:seen].t()) * scale
                    s.masked_fill_(hidden, -math.inf)
                    m = s.amax(-1, keepdim=True)
                    p = torch.exp(s - m)
                    z = p.sum(-1, keepdim=True)
                    out[head, r0:r1] = ((p @ vf[:seen]) / z).to(out.dtype)
                    if st["lse"] is not None:
                        w = c["lse_rows"]
                        first = max(r0, n - w)
                        if first < r1:
                            st["lse"][b, head, first - (n - w):r1 - (n - w)] = (m + torch.log(z))[first - r0:, 0]
        if st["lse"] is not None and n < c["lse_rows"]:
            st["lse"][b, :, :c["lse_rows"] - n] = -math.inf


def _plain_weighted(st):
    c = st["case"]
    G, scale = c["q_heads"] // c["kv_heads"], c["head_dim"] ** -0.5
    for b, n in enumerate(st["rows"]):
        st["kc"][b, :, n] = st["kn"][b]
        st["vc"][b, :, n] = st["vn"][b]
        st["tok"][b, :, n] = st["at"][b]
        k, v = st["kc"][b, :, :n + 1].float(), st["vc"][b, :, :n + 1].float()
        q = st["q"][b].float().view(c["kv_heads"], G, c["head_dim"])
        s = torch.matmul(q, k.transpose(1, 2).contiguous()) * scale
        p = torch.exp(s - s.amax(-1, keepdim=True))
        p = p / p.sum(-1, keepdim=True)
        st["out"][b] = torch.matmul(p, v).view(c["q_heads"], c["head_dim"])
        w = p.sum(1)
        st["weights"][b, :, :n] += w[:, :n]
        st["weights"][b, :, n] = w[:, n]


def _plain_evict(st):
    c = st["case"]
    keep = c["keep"]
    for b, n in enumerate(st["rows"]):
        if n <= keep:
            continue
        w, tok = st["weights"][b, :, :n], st["tok"][b, :, :n]
        recent = tok > tok.amax(-1, keepdim=True) - c["recent"]
        order = torch.sort(torch.where(recent, torch.full_like(w, math.inf), w), dim=-1, descending=True, stable=True).indices
        stays = torch.zeros((c["kv_heads"], n), dtype=torch.bool, device="cuda")
        stays.scatter_(1, order[:, :keep], True)
        # row i of the cut cache: itself if it stays, else the next kept row from past the budget
        late = torch.sort((~stays[:, keep:]).to(torch.int8), dim=-1, stable=True).indices + keep
        rank = (torch.cumsum(~stays[:, :keep], -1) - 1).clamp(0, n - keep - 1)
        source = torch.where(stays[:, :keep], torch.arange(keep, device="cuda")[None], late.gather(1, rank))
        for t in st["kc"] + st["vc"]:
            t[b, :, :keep] = t[b].gather(1, source[:, :, None].expand(-1, -1, c["head_dim"]))
        w[:, :keep] = w.gather(1, source)
        tok[:, :keep] = tok.gather(1, source)
        st["n"][b] = keep


def run(st):
    kind = st["case"]["kind"]
    W = _wkv() if own else None
    if kind == "rope":
        if own:
            W.wkv_rope(st["shape"], st["pos"], st["q"], st["q_out"], st["k"], st["k_out"])
        else:
            _plain_rope(st)
        return st["q_out"], st["k_out"]
    if kind == "prefill":
        if own:
            W.wkv_prefill_attention(st["shape"], st["q"], st["k"], st["v"], st["out"], st["lse"], st["ws"])
        else:
            _plain_prefill(st)
        return (st["out"],) if st["lse"] is None else (st["out"], st["lse"])
    if kind == "weighted":
        st["weights"].copy_(st["start"])             # the step adds to them: the same start for every pass
        if own:
            W.wkv_decode_step_weighted(st["shape"], st["q"], st["kn"], st["vn"], st["kc"], st["vc"], st["n"], st["weights"],
                                       st["tok"], st["at"], st["out"], st["ws"])
        else:
            _plain_weighted(st)
        return st["out"], st["weights"], st["tok"], st["kc"], st["vc"]
    # (the caches come out the same from a second pass: the rows that move are not written to)
    st["state"].copy_(st["first"])
    if own:
        W.wkv_cache_evict(st["shape"], st["kc"], st["vc"], st["weights"], st["tok"], st["n"], st["keep"], st["case"]["recent"], st["ws"])
    else:
        _plain_evict(st)
    return [st["weights"], st["tok"], st["n"]] + st["kc"] + st["vc"]


def work(case):
    d, kv = case["head_dim"], case["kv_heads"]
    e = 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "rope":
        tokens = sum(_ints(case["lens"]))
        heads = case["q_heads"] + kv
        return {"bytes": tokens * (2 * heads * d * e + 4), "flops": tokens * heads * case["rotary"] * 3}
    if case["kind"] == "prefill":
        lens, past, q = _ints(case["lens"]), _ints(case["past"]), case["q_heads"]
        pairs = sum(n * p + n * (n + 1) // 2 for n, p in zip(lens, past))
        rows, keys = sum(lens), sum(lens) + sum(past)
        return {"bytes": (2 * rows * q + 2 * keys * kv) * d * e + 4 * len(lens) * q * case["lse_rows"], "flops": 4 * d * q * pairs}
    rows = _ints(case["rows"])
    if case["kind"] == "weighted":
        n, q = sum(rows) + len(rows), case["q_heads"]
        # rows of the caches, weights read and written, the new rows written, queries, outputs
        return {"bytes": n * kv * (2 * d * e + 8) + len(rows) * (2 * kv * d * e + q * d * (e + 4)), "flops": 4 * n * q * d}
    # weights and positions; what moves depends on the weights: a row that stays lies past the budget with the
    # chance of that place, (n - keep) / n
    moved = sum(case["keep"] * (n - case["keep"]) / n for n in rows if n > case["keep"])
    return {"bytes": int(sum(rows) * kv * 8 + moved * kv * (4 * case["layers"] * d * e + 8)), "flops": sum(rows) * kv}


# ---- the definition in 64 bits --------------------------------------------------------------------------------------

def _exact_rope(st):
    c = st["case"]
    r = c["rotary"]
    first = torch.arange(r // 2, device="cuda") * (2 if c["interleaved"] else 1)
    second = first + (1 if c["interleaved"] else r // 2)
    turn = torch.polar(torch.full_like(st["inv"], st["amp"]), torch.zeros_like(st["inv"]))
    results = []
    for x, out, cache in ((st["q"], st["q_out"], False), (st["k"], st["k_out"], True)):
        y = out.double().clone()
        for b in range(x.shape[0]):
            tokens = torch.nonzero(st["pos"][b] >= 0)[:, 0]
            z = x[b, tokens].double()
            angle = st["pos"][b, tokens].double()[:, None] * st["inv"][None]
            w = torch.complex(z[..., first], z[..., second]) * (torch.polar(torch.ones_like(angle), angle) * turn)[:, None]
            z[..., first], z[..., second] = w.real, w.imag
            if cache:
                y[b][:, tokens] = z.transpose(0, 1)
            else:
                y[b, tokens] = z
        results.append(y)
    return tuple(results)


def _exact_prefill(st):
    c = st["case"]
    lens, past = _ints(c["lens"]), _ints(c["past"])
    total = [n + p for n, p in zip(lens, past)]
    G, keep = c["q_heads"] // c["kv_heads"], c["lse_rows"]
    out = torch.zeros_like(st["out"], dtype=torch.float64)
    lse = torch.full((len(lens), c["q_heads"], keep), -math.inf, dtype=torch.float64, device="cuda")
    box = dict(st, out=out)
    for b, n in enumerate(lens):
        q, o, k, v = _rows_of(box, b, lens, total, c["layout"] == "packed")
        for head in range(c["q_heads"]):
            k64, v64 = k[head // G].double(), v[head // G].double()
            for r0 in range(0, n, 2048):
                r1 = min(n, r0 + 2048)
                logits = q[head, r0:r1].double() @ k64[:past[b] + r1].t()
                logits /= math.sqrt(c["head_dim"])
                logits[:, past[b] + r0:] += torch.full((r1 - r0, r1 - r0), -math.inf, dtype=torch.float64, device="cuda").triu(1)
                norm = torch.logsumexp(logits, -1)
                o[head, r0:r1] = torch.exp(logits - norm[:, None]) @ v64[:past[b] + r1]
                first = max(r0, n - keep)
                if first < r1:
                    lse[b, head, first - (n - keep):r1 - (n - keep)] = norm[first - r0:]
    return (out, lse) if keep else (out,)


def _exact_weighted(st):
    c = st["case"]
    G = c["q_heads"] // c["kv_heads"]
    out, weights = torch.zeros_like(st["out"], dtype=torch.float64), st["start"].double()
    tok, kc, vc = st["tok"].clone(), st["kc"].clone(), st["vc"].clone()
    for b, n in enumerate(st["rows"]):
        for h in range(c["kv_heads"]):
            kc[b, h, n], vc[b, h, n], tok[b, h, n] = st["kn"][b, h], st["vn"][b, h], st["at"][b]
            logits = kc[b, h, :n + 1].double() @ st["q"][b, h * G:(h + 1) * G].double().t() / math.sqrt(c["head_dim"])
            share = torch.softmax(logits, 0)
            out[b, h * G:(h + 1) * G] = share.t() @ vc[b, h, :n + 1].double()
            weights[b, h, n] = 0.0
            weights[b, h, :n + 1] += share.sum(1)
    return out, weights, tok, kc, vc


def _exact_evict(st):
    import numpy as np
    c = st["case"]
    keep = c["keep"]
    weights, tok, n = st["weights"].clone(), st["tok"].clone(), st["n"].clone()
    caches = [t.clone() for t in st["kc"] + st["vc"]]
    for b, rows in enumerate(st["rows"]):
        for h in range(c["kv_heads"] if rows > keep else 0):
            w, t = weights[b, h, :rows].cpu().numpy(), tok[b, h, :rows].cpu().numpy()
            old = t.astype(np.int64) <= int(t.max()) - c["recent"]
            # protected rows first, then the heavier, then the lower row
            order = np.lexsort((np.arange(rows), -w.astype(np.float64), old))
            kept = np.sort(order[:keep])
            late, holes = kept[kept >= keep], np.setdiff1d(np.arange(keep), kept)
            src, dst = torch.from_numpy(late).cuda(), torch.from_numpy(holes).cuda()
            for x in caches + [weights, tok]:
                x[b, h, dst] = x[b, h, src]
            n[b, h] = keep
    return [weights, tok, n] + caches


def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    return {"rope": _exact_rope, "prefill": _exact_prefill, "weighted": _exact_weighted, "evict": _exact_evict}[case["kind"]](st)
