"""The operators of generation over a compact KV cache and the calls they are measured by: normalised queries and keys with
rotary positions of one or several axes, caches held in 8 or 4 bits with the decode step that reads them, and attention for
a tree of drafted tokens with the acceptance of one of its paths.

A case is a dict of plain values.  ``kind`` names the operator:

norm_rope  ``wkv_norm_rope``: queries and keys of ``lens`` tokens a sequence (padded to the longest), read from the rows of one
           fused projection [batch, token, (q | k | v) heads, channel], normalised a head at a time (``norm``) and turned by
           positions on ``axes`` axes, keys written into a cache [batch, head, row, channel].
store      ``wkv_cache_quantize``, then ``wkv_cache_dequantize`` of the rows written: ``rows`` rows a sequence and KV head
           in ``layers`` layers, behind ``behind`` rows that the caches hold already.  ``source`` is the number of rows they
           are picked from by ascending positions, as the window selection leaves them (0: the rows as they lie).
step       ``wkv_decode_step_quantized``: one token over caches of ``rows`` rows (one number a sequence) in ``format``; the
           new token's row is read back.
tree       ``wkv_decode_tree`` in ``layers`` layers that share their row counts, then ``wkv_tree_accept`` of a path in all of
           them: ``nodes`` drafted tokens over caches of ``rows`` rows.

Formats: "e4m3" (8 bits) and "e2m1" (4 bits), with a power of two for every 32 channels of a row.  What a cache holds is compared as the
values that codes and scales stand for.  Where ``own`` is false, ``run`` computes an operator from elementary torch operations in 32 bits
(angles in 64).
"""
import math
import random

import torch

own = False

_TORCH = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_ROOM = 256              # rows a cache has for tokens to come
_EPS = 1e-6
_GROUP = 32              # channels that share a scale
_LEAST = -100            # exponent of the smallest scale


def _wkv():
    import paper_2503_17922_amd as W
    return W


def _dtype(W, name):
    return {"bf16": W.WKV_BF16, "f16": W.WKV_F16, "f32": W.WKV_F32}[name]


def _format(W, name):
    return {"e4m3": W.WKV_CACHE_E4M3, "e2m1": W.WKV_CACHE_E2M1}[name]


def _ints(text):
    return [int(x) for x in str(text).split()]


def _text(xs):
    return " ".join(str(x) for x in xs)


def _norm_rope(name, lens, **kw):
    c = dict(name=name, kind="norm_rope", dtype="bf16", q_heads=32, kv_heads=8, head_dim=128, rotary=128, interleaved=False,
             norm=True, axes=1, lens=_text(lens), first=0, theta=500000.0)
    c.update(kw)
    return c


def _store(name, rows, **kw):
    c = dict(name=name, kind="store", dtype="bf16", format="e4m3", kv_heads=8, head_dim=128, layers=4, rows=_text(rows), source=0,
             behind=0)
    c.update(kw)
    return c


def _step(name, rows, **kw):
    c = dict(name=name, kind="step", dtype="bf16", format="e4m3", q_heads=32, kv_heads=8, head_dim=128, rows=_text(rows))
    c.update(kw)
    return c


def _tree(name, rows, **kw):
    c = dict(name=name, kind="tree", dtype="bf16", q_heads=32, kv_heads=8, head_dim=128, layers=1, nodes=16, rows=_text(rows))
    c.update(kw)
    return c


_MIXED = [4128, 2080, 544, 3001, 777, 4500, 1234, 96, 2600, 3999, 1777]


def listed():
    return [
        # the new token of each of 64 sequences that generate together: latency
        _norm_rope("norm_rope_step_64", [1] * 64, first=4096),
        # the prompt of the 32K benchmark in a model that normalises queries and keys
        _norm_rope("norm_rope_prompt_32k", [32768]),
        # video prompts of odd lengths: time, height and width of a patch, interleaved pairs, half precision
        _norm_rope("norm_rope_video_f16", [9973, 2051, 5003], dtype="f16", q_heads=28, kv_heads=4, interleaved=True, axes=3, theta=10000.0),
        # the new token's row of each of 64 sequences, all layers of a group: latency
        _store("store_step_64", [1] * 64, behind=4128),
        # the rows that the window selection keeps of the 32K benchmark's prompt, from the full caches into 8 bits
        _store("store_kept_32k", [4128], source=32768),
        # prompts of different lengths into 4 bits, half precision
        _store("store_ragged_e2m1", [9973, 2051, 1, 5003, 377], format="e2m1", dtype="f16", kv_heads=4, layers=2),
        # one user's token over a compact cache in 8 bits: latency
        _step("step_1", [4128]),
        # generation at full batch over caches in 8 bits
        _step("step_64", [4128] * 64),
        # mixed lengths in 4 bits, seven query heads to a KV head, half precision
        _step("step_mixed_e2m1", _MIXED * 4, format="e2m1", dtype="f16", q_heads=28, kv_heads=4),
        # one user's drafted tree over the compact caches of a layer group: latency
        _tree("tree_1", [4128], layers=4),
        # trees at full batch
        _tree("tree_64", [4128] * 64),
        # the largest trees over mixed lengths, seven query heads to a KV head, half precision
        _tree("tree_mixed_f16", _MIXED, nodes=64, dtype="f16", q_heads=28, kv_heads=4),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_HEADS = {64: [(64, 8), (28, 4), (12, 2), (32, 32)], 128: [(32, 8), (32, 8), (64, 8), (28, 4), (12, 2), (32, 32)]}


def draw(rng):
    kind = rng.choice(["norm_rope", "store", "step", "tree"])
    d = rng.choice([64, 128, 128])
    q, kv = rng.choice(_HEADS[d])
    c = dict(kind=kind, dtype=rng.choice(["bf16"] * 5 + ["f16"] * 3 + ["f32"]), q_heads=q, kv_heads=kv, head_dim=d)
    if kind == "norm_rope":
        batch = _log(rng, 1, 64)
        longest = _log(rng, 1, 16384 // batch)
        c.update(rotary=rng.choice([d, d, d // 2]), interleaved=rng.random() < 0.4, norm=rng.random() < 0.8, axes=rng.choice([1, 1, 2, 3, 4]),
                 first=rng.choice([0, 0, _log(rng, 1, 100000)]), theta=rng.choice([10000.0, 500000.0, 1000000.0]),
                 lens=_text([longest] + [_log(rng, max(1, longest // 8), longest) for _ in range(batch - 1)]))
    elif kind == "store":
        batch = _log(rng, 1, 32)
        longest = _log(rng, 1, 16384 // batch)
        rows = [longest] + [_log(rng, max(1, longest // 8), longest) for _ in range(batch - 1)]
        c.update(format=rng.choice(["e4m3", "e2m1"]), layers=rng.choice([1, 2, 4]), rows=_text(rows),
                 source=rng.choice([0, longest * rng.choice([1, 2, 4])]), behind=rng.choice([0, _log(rng, 1, 1000)]))
        del c["q_heads"]
    elif kind == "step":
        batch = _log(rng, 1, 48)
        longest = _log(rng, 64, 16384) // (1 + batch // 8) + 1
        c.update(format=rng.choice(["e4m3", "e2m1"]), rows=_text([longest] + [_log(rng, max(1, longest // 8), longest) for _ in range(batch - 1)]))
    else:
        batch = _log(rng, 1, 32)
        longest = _log(rng, 64, 16384 if c["dtype"] != "f32" else 4096) // (1 + batch // 8) + 1
        c.update(layers=rng.choice([1, 2]), nodes=_log(rng, 1, 64), rows=_text([longest] + [_log(rng, max(1, longest // 8), longest) for _ in range(batch - 1)]))
    return c


# ---- caches in 8 and 4 bits -----------------------------------------------------------------------------------------

_MAGNITUDES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]      # of an e2m1 code


def _power(e):
    """2^e for whole numbers e from -126 to 127, by its bits (a power function may be a step off)."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _quantized(x, fmt):
    """x [..., d] as numbers of the format and the exponents of their scales [..., d / 32]: the smallest power of two with which
    no magnitude exceeds the format's largest, 1.75 * 2^8 or 1.5 * 2^2; each number to the nearest, ties to the even."""
    parts = x.float().unflatten(-1, (-1, _GROUP))
    most = parts.abs().amax(-1)
    fraction, exponent = torch.frexp(most)                    # most = fraction * 2^exponent, fraction from 1/2 to 1
    scale = (exponent - 9 + (fraction > 0.875)) if fmt == "e4m3" else (exponent - 3 + (fraction > 0.75))
    scale = torch.where(most > 0, scale, _LEAST).clamp(min=_LEAST)
    y = parts * _power(-scale)[..., None]
    least, bits = (-6, 3) if fmt == "e4m3" else (0, 1)        # of a normal number, of its fraction
    step = torch.frexp(y.abs())[1] - 1
    step = torch.where(y != 0, step, least).clamp(min=least) - bits
    return torch.round(y * _power(-step)) * _power(step), scale


def _values(numbers, scale, dtype):
    v = (numbers * _power(scale)[..., None]).flatten(-2)
    return (v.clamp(-65504.0, 65504.0) if dtype == "f16" else v).to(_TORCH[dtype])


def _codes(numbers, scale, fmt):
    """The bytes that hold them: e4m3 a byte each, e2m1 two to a byte, the even channel in the lower half; scales biased by 127."""
    n = numbers.flatten(-2)
    if fmt == "e4m3":
        codes = n.to(torch.float8_e4m3fn).view(torch.uint8)
    else:
        edges = torch.tensor(_MAGNITUDES, device=n.device)
        half = torch.bucketize(n.abs(), edges) + 8 * torch.signbit(n)
        codes = (half[..., 0::2] + 16 * half[..., 1::2]).to(torch.uint8)
    return codes, (scale + 127).to(torch.uint8)


def _held(codes, scales, fmt):
    """The values [..., d] that codes and scales stand for, in 32 bits."""
    if fmt == "e4m3":
        n = codes.view(torch.float8_e4m3fn).float()
    else:
        table = torch.tensor(_MAGNITUDES + [-m for m in _MAGNITUDES], device=codes.device)
        n = torch.stack([table[(codes & 15).int()], table[(codes >> 4).int()]], -1).flatten(-2)
    return (n.unflatten(-1, (-1, _GROUP)) * _power(scales.int() - 127)[..., None]).flatten(-2)


# ---- inputs ---------------------------------------------------------------------------------------------------------

def _normal(g, shape, dtype, scale=1.0):
    return (torch.randn(shape, device="cuda", dtype=torch.float32, generator=g) * scale).to(_TORCH[dtype])


def _keys(g, shape, dtype):
    """Rows as keys are: a few channels of a head several times as large as the others."""
    x = torch.randn(shape, device="cuda", dtype=torch.float32, generator=g)
    x *= torch.exp(0.7 * torch.randn((1, shape[1], 1, shape[3]), device="cuda", generator=g))
    return x.to(_TORCH[dtype])


def _axis_of_pair(case):
    """Axis of every pair of channels: one run of pairs an axis."""
    pairs, axes = case["rotary"] // 2, case["axes"]
    return [min(i * axes // pairs, axes - 1) for i in range(pairs)]


def _counts(rows, kv):
    return torch.tensor(rows, dtype=torch.int32, device="cuda")[:, None].repeat(1, kv)


def _trees(rng, batch, nodes):
    """Parents (-1: the last row of the cache) and a path from the top of the tree, with how much of it was accepted."""
    parents, paths, accepted = [], [], []
    for _ in range(batch):
        p = [rng.randrange(max(-1, t - 8), t) if rng.random() < 0.7 else t - 1 for t in range(nodes)]
        at, path = rng.randrange(nodes), []
        while at >= 0:
            path.append(at)
            at = p[at]
        path.reverse()
        parents.append(p)
        accepted.append(rng.randrange(len(path) + 1))
        paths.append(path + [-1] * (nodes - len(path)))
    return parents, paths, accepted


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    d, kv, dt, kind = case["head_dim"], case["kv_heads"], case["dtype"], case["kind"]
    st = dict(case=case)
    W = _wkv() if own else None
    if kind == "norm_rope":
        lens, q, axes = _ints(case["lens"]), case["q_heads"], case["axes"]
        B, T, h = len(lens), max(lens), q + 2 * kv
        # (projected rows of very different sizes, as normalisation finds them)
        rows = (torch.randn((B, T, h, d), device="cuda", generator=g) * torch.exp(torch.randn((B, T, h, 1), device="cuda", generator=g))).to(_TORCH[dt])
        pos = torch.full((B, T, axes), -1, dtype=torch.int32, device="cuda")       # padding
        for b, n in enumerate(lens):
            at = torch.arange(n, device="cuda", dtype=torch.int32) + case["first"] + 7 * b
            # frames of 24 x 40 patches: time, then height and width (and the token's own number on a fourth axis)
            pos[b, :n] = torch.stack([at if axes == 1 else at // 960, at // 40 % 24, at % 40, at], -1)[:, :axes]
        inv = [case["theta"] ** (-2.0 * i / case["rotary"]) for i in range(case["rotary"] // 2)]
        axis = _axis_of_pair(case)
        st.update(q=rows[:, :, :q], k=rows[:, :, q:q + kv], pos=pos, axis=torch.tensor(axis, device="cuda"),
                  inv=torch.tensor(inv, dtype=torch.float64, device="cuda"),
                  qw=(1.0 + 0.3 * torch.randn(d, device="cuda", generator=g)).to(_TORCH[dt]) if case["norm"] else None,
                  kw=(1.0 + 0.3 * torch.randn(d, device="cuda", generator=g)).to(_TORCH[dt]) if case["norm"] else None,
                  q_out=torch.zeros((B, T, q, d), dtype=_TORCH[dt], device="cuda"),
                  k_out=torch.zeros((B, kv, T + _ROOM, d), dtype=_TORCH[dt], device="cuda"))
        if own:
            st["shape"] = W.NormRopeShape(batch=B, n_tokens=T, n_q_heads=q, n_kv_heads=kv, head_dim=d, dtype=_dtype(W, dt), inv_freq=inv,
                                          n_axes=axes, axis_of_pair=axis, eps=_EPS, interleaved=case["interleaved"],
                                          q_strides=(T * h * d, d, h * d), k_strides=(T * h * d, d, h * d),
                                          q_out_strides=(T * q * d, d, q * d), k_out_strides=(kv * (T + _ROOM) * d, (T + _ROOM) * d, d))
        return st
    rows = _ints(case["rows"])
    B, most = len(rows), max(rows)
    if kind == "store":
        source, layers, behind = case["source"], case["layers"], case["behind"]
        size = max(source, most)
        st.update(k=[_keys(g, (B, kv, size, d), dt) for _ in range(layers)], v=[_normal(g, (B, kv, size, d), dt) for _ in range(layers)],
                  n=_counts(rows, kv), first=_counts([behind] * B, kv), end=_counts([behind + n for n in rows], kv), tok=None,
                  k_out=[torch.zeros((B, kv, most, d), dtype=_TORCH[dt], device="cuda") for _ in range(layers)],
                  v_out=[torch.zeros((B, kv, most, d), dtype=_TORCH[dt], device="cuda") for _ in range(layers)])
        if source:
            tok = torch.rand((B, kv, source), device="cuda", generator=g).argsort(-1)[..., :most]
            # (each sequence's own number of ascending positions, padded with -1)
            here = torch.arange(most, device="cuda") < st["n"][..., None]
            tok = torch.where(here, tok, source).sort(-1).values
            st["tok"] = torch.where(here, tok, -1).to(torch.int32)
        cap = behind + most + _ROOM
        per_row = d if case["format"] == "e4m3" else d // 2
        for name in "kv":
            st[name + "_codes"] = [torch.zeros((B, kv, cap, per_row), dtype=torch.uint8, device="cuda") for _ in range(layers)]
            st[name + "_scales"] = [torch.zeros((B, kv, cap, d // _GROUP), dtype=torch.uint8, device="cuda") for _ in range(layers)]
        if own:
            st["shape"] = W.QuantizedShape(batch=B, n_kv_heads=kv, head_dim=d, dtype=_dtype(W, dt), format=_format(W, case["format"]), capacity=cap,
                                           n_rows=most, row_capacity=size)
            st["back"] = W.QuantizedShape(batch=B, n_kv_heads=kv, head_dim=d, dtype=_dtype(W, dt), format=_format(W, case["format"]), capacity=cap,
                                          n_rows=most)
        return st
    q, cap = case["q_heads"], most + _ROOM
    if kind == "step":
        st.update(q=_normal(g, (B, q, d), dt, 1.5), kn=_keys(g, (B, kv, 1, d), dt)[:, :, 0], vn=_normal(g, (B, kv, d), dt), n=_counts(rows, kv),
                  out=torch.empty((B, q, d), device="cuda"),
                  row=[torch.zeros((B, kv, 1, d), dtype=_TORCH[dt], device="cuda") for _ in range(2)])
        for name, made in (("k", _keys), ("v", _normal)):
            st[name + "_codes"], st[name + "_scales"] = _codes(*_quantized(made(g, (B, kv, cap, d), dt), case["format"]), case["format"])
        if own:
            kw = dict(batch=B, n_q_heads=q, n_kv_heads=kv, head_dim=d, dtype=_dtype(W, dt), format=_format(W, case["format"]), capacity=cap)
            st["shape"] = W.QuantizedShape(flags=W.WKV_DECODE_KEEP_COUNT, **kw)
            st["back"] = W.QuantizedShape(n_rows=1, **kw)
            st["ws"] = torch.empty(W.wkv_decode_quantized_workspace_bytes(st["shape"]), dtype=torch.uint8, device="cuda")
        return st
    T, layers = case["nodes"], case["layers"]
    parents, paths, accepted = _trees(random.Random(seed), B, T)
    h = q + 2 * kv
    # (logits of a standard deviation of 1.5)
    new = [torch.cat([_normal(g, (B, T, q, d), dt, 1.5), _normal(g, (B, T, 2 * kv, d), dt)], 2) for _ in range(layers)]
    st.update(q=[x[:, :, :q] for x in new], kn=[x[:, :, q:q + kv] for x in new], vn=[x[:, :, q + kv:] for x in new],
              kc=[_normal(g, (B, kv, cap, d), dt) for _ in range(layers)], vc=[_normal(g, (B, kv, cap, d), dt) for _ in range(layers)],
              parent=torch.tensor(parents, dtype=torch.int32, device="cuda"), path=torch.tensor(paths, dtype=torch.int32, device="cuda"),
              accepted=torch.tensor(accepted, dtype=torch.int32, device="cuda"), first=_counts(rows, kv), n=_counts(rows, kv),
              out=[torch.zeros((B, T, q, d), dtype=_TORCH[dt], device="cuda") for _ in range(layers)])
    if own:
        st["shape"] = W.TreeShape(batch=B, n_q_heads=q, n_kv_heads=kv, head_dim=d, dtype=_dtype(W, dt), n_nodes=T, capacity=cap,
                                  q_strides=(T * h * d, d, h * d), new_strides=(T * h * d, d, h * d), out_strides=(T * q * d, d, q * d))
        st["ws"] = torch.empty(W.wkv_tree_workspace_bytes(st["shape"]), dtype=torch.uint8, device="cuda")
    return st


# ---- one pass -------------------------------------------------------------------------------------------------------

def _normed(x, weight):
    y = x.float()
    return y if weight is None else y * torch.rsqrt((y * y).mean(-1, keepdim=True) + _EPS) * weight.float()


def _turn(y, cos, sin, case, dtype):
    """Pairs of the first ``rotary`` channels of y [B, T, H, d] turned by angles given as cos and sin [B, T, 1, rotary / 2]."""
    r = case["rotary"]
    if case["interleaved"]:
        a, b = y[..., 0:r:2], y[..., 1:r:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = y[..., :r // 2], y[..., r // 2:r]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turned, y[..., r:]], -1).to(dtype)


def _plain_norm_rope(st):
    c = st["case"]
    T, dtype = st["pos"].shape[1], st["q"].dtype
    angle = (st["pos"][:, :, st["axis"]].double() * st["inv"])[:, :, None]
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    valid = (st["pos"] >= 0).all(-1)[:, :, None, None]
    st["q_out"].copy_(torch.where(valid, _turn(_normed(st["q"], st["qw"]), cos, sin, c, dtype), st["q_out"]))
    k_rows = st["k_out"][:, :, :T].transpose(1, 2)
    k_rows.copy_(torch.where(valid, _turn(_normed(st["k"], st["kw"]), cos, sin, c, dtype), k_rows))


def _plain_store(st):
    c = st["case"]
    most = st["k_out"][0].shape[2]
    here = (torch.arange(most, device="cuda") < st["n"][..., None])[..., None]
    for x, out in zip(st["k"] + st["v"], st["k_out"] + st["v_out"]):
        rows = x[:, :, :most] if st["tok"] is None else x.gather(2, st["tok"].clamp(min=0).long()[..., None].expand(-1, -1, -1, c["head_dim"]))
        out.copy_(torch.where(here, _values(*_quantized(rows, c["format"]), c["dtype"]), out))


def _attend(q, k, v, hidden, scale):
    """q [B, H, R, d] over k, v [B, H, n, d] in 32 bits, without the pairs that are hidden [B, H or 1, R or 1, n]."""
    s = torch.matmul(k, q.transpose(2, 3).contiguous()).transpose(2, 3) * scale
    s = s.masked_fill(hidden, -math.inf)
    p = torch.exp(s - s.amax(-1, keepdim=True))
    return torch.matmul(p, v) / p.sum(-1, keepdim=True)


def _plain_step(st):
    c = st["case"]
    B, kv, d = st["kn"].shape
    G, fmt = c["q_heads"] // kv, c["format"]
    at = st["n"].long()[..., None]
    held = {}
    for name, new, row in (("k", st["kn"], st["row"][0]), ("v", st["vn"], st["row"][1])):
        numbers, scale = _quantized(new, fmt)
        codes, scales = _codes(numbers, scale, fmt)
        for cache, x in ((st[name + "_codes"], codes), (st[name + "_scales"], scales)):
            cache.scatter_(2, at[..., None].expand(-1, -1, 1, x.shape[-1]), x[:, :, None])
        row[:, :, 0] = _values(numbers, scale, c["dtype"])
        held[name] = _held(st[name + "_codes"], st[name + "_scales"], fmt)
    hidden = torch.arange(held["k"].shape[2], device="cuda") > st["n"][..., None]
    st["out"].copy_(_attend(st["q"].float().view(B, kv, G, d), held["k"], held["v"], hidden[:, :, None], d ** -0.5).view(B, kv * G, d))


def _plain_tree(st):
    c = st["case"]
    B, T, kv, d = st["kn"][0].shape
    G, cap = c["q_heads"] // kv, st["kc"][0].shape[2]
    n = st["n"].long()
    at = n[..., None] + torch.arange(T, device="cuda")                        # [B, kv, T]: the nodes' rows
    # a node's ancestors and itself: the paths of parents of any length
    up = torch.arange(T, device="cuda") == st["parent"][..., None]
    family = torch.matrix_power(torch.eye(T, device="cuda", dtype=torch.float64) + up.double(), 64) > 0
    seen = torch.zeros((B, kv, T, cap), dtype=torch.bool, device="cuda")
    seen.scatter_(3, at[:, :, None].expand(-1, -1, T, -1), family[:, None].expand(-1, kv, -1, -1))
    hidden = ~(seen | (torch.arange(cap, device="cuda") < n[..., None])[:, :, None]).repeat_interleave(G, 2)
    for q, kn, vn, kc, vc, out in zip(st["q"], st["kn"], st["vn"], st["kc"], st["vc"], st["out"]):
        for cache, new in ((kc, kn), (vc, vn)):
            cache.scatter_(2, at[..., None].expand(-1, -1, -1, d), new.transpose(1, 2))
        rows = q.float().unflatten(2, (kv, G)).permute(0, 2, 1, 3, 4).reshape(B, kv, T * G, d)
        o = _attend(rows, kc.float(), vc.float(), hidden, d ** -0.5)
        out.copy_(o.view(B, kv, T, G, d).permute(0, 2, 1, 3, 4).reshape(B, T, kv * G, d))
    source = (n[..., None] + st["path"].clamp(min=0).long()[:, None])[..., None].expand(-1, -1, -1, d)
    taken = (torch.arange(T, device="cuda") < st["accepted"][:, None])[:, None, :, None]
    to = at[..., None].expand(-1, -1, -1, d)
    for cache in st["kc"] + st["vc"]:
        cache.scatter_(2, to, torch.where(taken, cache.gather(2, source), cache.gather(2, to)))
    st["n"] += st["accepted"][:, None]


def run(st):
    kind = st["case"]["kind"]
    W = _wkv() if own else None
    if kind == "norm_rope":
        if own:
            W.wkv_norm_rope(st["shape"], st["pos"], st["qw"], st["kw"], st["q"], st["q_out"], st["k"], st["k_out"])
        else:
            _plain_norm_rope(st)
        return st["q_out"], st["k_out"]
    if kind == "store":
        if own:
            W.wkv_cache_quantize(st["shape"], st["k"], st["v"], st["tok"], st["n"], st["first"], st["k_codes"], st["k_scales"], st["v_codes"],
                                 st["v_scales"])
            W.wkv_cache_dequantize(st["back"], st["k_codes"], st["k_scales"], st["v_codes"], st["v_scales"], st["first"], st["end"],
                                   st["k_out"], st["v_out"])
        else:
            _plain_store(st)
        return st["k_out"] + st["v_out"]
    if kind == "step":
        if own:
            W.wkv_decode_step_quantized(st["shape"], st["q"], st["kn"], st["vn"], st["k_codes"], st["k_scales"], st["v_codes"], st["v_scales"],
                                        st["n"], st["out"], st["ws"])
            W.wkv_cache_dequantize(st["back"], [st["k_codes"]], [st["k_scales"]], [st["v_codes"]], [st["v_scales"]], st["n"], None,
                                   st["row"][:1], st["row"][1:])
        else:
            _plain_step(st)
        return [st["out"]] + st["row"]
    st["n"].copy_(st["first"])                   # the acceptance adds to it: the same start for every pass
    if own:
        for layer in zip(st["q"], st["kn"], st["vn"], st["kc"], st["vc"], st["out"]):
            q, kn, vn, kc, vc, out = layer
            W.wkv_decode_tree(st["shape"], q, kn, vn, st["parent"], kc, vc, st["n"], out, st["ws"])
        W.wkv_tree_accept(st["shape"], st["kc"], st["vc"], st["path"], st["accepted"], st["n"])
    else:
        _plain_tree(st)
    return [st["n"]] + st["out"] + st["kc"] + st["vc"]


def work(case):
    d, kv = case["head_dim"], case["kv_heads"]
    e = 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "norm_rope":
        tokens = sum(_ints(case["lens"]))
        heads = case["q_heads"] + kv
        return {"bytes": tokens * (2 * heads * d * e + 4 * case["axes"]) + (2 * d * e if case["norm"] else 0),
                "flops": tokens * heads * (case["rotary"] * 3 + (4 * d if case["norm"] else 0))}
    rows = _ints(case["rows"])
    if case["kind"] == "store":
        held = (d if case["format"] == "e4m3" else d // 2) + d // _GROUP
        units = 2 * case["layers"] * kv * sum(rows)
        # rows read, what is held written and read, rows written; positions
        return {"bytes": units * (2 * d * e + 2 * held) + (4 * kv * sum(rows) if case["source"] else 0), "flops": units * d * 4}
    q = case["q_heads"]
    if case["kind"] == "step":
        held = (d if case["format"] == "e4m3" else d // 2) + d // _GROUP
        n = sum(rows) + len(rows)
        # what is held of the rows, the new ones read, written and read back, queries, outputs
        return {"bytes": 2 * n * kv * held + len(rows) * (4 * kv * d * e + q * d * (e + 4)), "flops": 4 * n * q * d}
    T, layers = case["nodes"], case["layers"]
    new = len(rows) * T
    # rows of the caches, the nodes' rows read and written, queries, outputs; an accepted path (half the depth of a tree) is small beside them
    return {"bytes": layers * (2 * sum(rows) * kv * d * e + new * (4 * kv + 2 * q) * d * e), "flops": layers * 4 * d * q * T * (sum(rows) + len(rows))}


# ---- the definition in 64 bits --------------------------------------------------------------------------------------

def _exact_norm_rope(st):
    c = st["case"]
    r = c["rotary"]
    pair = torch.arange(r // 2, device="cuda")
    first, second = (2 * pair, 2 * pair + 1) if c["interleaved"] else (pair, pair + r // 2)
    results = []
    for x, weight, out, cache in ((st["q"], st["qw"], st["q_out"], False), (st["k"], st["kw"], st["k_out"], True)):
        y = out.double().clone()
        for b in range(x.shape[0]):
            tokens = torch.nonzero(st["pos"][b].amin(-1) >= 0)[:, 0]
            z = x[b, tokens].double()
            if weight is not None:
                z = z / torch.sqrt(z.square().sum(-1, keepdim=True) / z.shape[-1] + _EPS) * weight.double()
            angle = st["pos"][b, tokens].double().index_select(1, st["axis"]) * st["inv"][None]
            w = torch.complex(z[..., first], z[..., second]) * torch.polar(torch.ones_like(angle), angle)[:, None]
            z[..., first], z[..., second] = w.real, w.imag
            if cache:
                y[b][:, tokens] = z.transpose(0, 1)
            else:
                y[b, tokens] = z
        results.append(y)
    return tuple(results)


def _nearest(x, fmt):
    """The definition, from the list of a format's numbers: x [..., d] in 64 bits, rounded."""
    if fmt == "e4m3":
        numbers = [m * 2.0 ** -9 for m in range(8)] + [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8)][:-1]
    else:
        numbers = _MAGNITUDES
    table = torch.tensor(numbers, dtype=torch.float64, device="cuda")
    parts = x.double().reshape(-1, _GROUP)
    most = parts.abs().amax(-1)
    scale = torch.full_like(most, 2.0 ** _LEAST)
    for e in range(_LEAST, 20):                                 # the smallest that holds the largest
        scale = torch.where(most > table[-1] * 2.0 ** e, 2.0 ** (e + 1), scale)
    scale = scale[:, None]
    y = (parts / scale).abs()
    above = torch.searchsorted(table, y).clamp(max=len(numbers) - 1)
    below = (above - 1).clamp(min=0)
    lo, hi = y - table[below], table[above] - y
    index = torch.where(lo < hi, below, torch.where(lo > hi, above, torch.where(below % 2 == 0, below, above)))
    return (torch.sign(parts) * table[index] * scale).reshape(x.shape)


def _exact_store(st):
    c = st["case"]
    results = []
    for x, out in zip(st["k"] + st["v"], st["k_out"] + st["v_out"]):
        y = out.double().clone()
        for b, n in enumerate(_ints(c["rows"])):
            for h in range(c["kv_heads"]):
                rows = x[b, h, :n] if st["tok"] is None else x[b, h].index_select(0, st["tok"][b, h, :n].long())
                y[b, h, :n] = _nearest(rows, c["format"])
        results.append(y)
    return results


def _exact_step(st):
    c = st["case"]
    G = c["q_heads"] // c["kv_heads"]
    out = torch.zeros_like(st["out"], dtype=torch.float64)
    kn, vn = _nearest(st["kn"], c["format"]), _nearest(st["vn"], c["format"])
    for b, n in enumerate(_ints(c["rows"])):
        k, v = (torch.cat([_held(st[x + "_codes"][b, :, :n], st[x + "_scales"][b, :, :n], c["format"]).double(), new[b][:, None]], 1)
                for x, new in (("k", kn), ("v", vn)))
        for h in range(c["kv_heads"]):
            logits = k[h] @ st["q"][b, h * G:(h + 1) * G].double().t() / math.sqrt(c["head_dim"])
            out[b, h * G:(h + 1) * G] = torch.softmax(logits, 0).t() @ v[h]
    return [out, kn[:, :, None], vn[:, :, None]]


def _exact_tree(st):
    c = st["case"]
    G, T, rows = c["q_heads"] // c["kv_heads"], c["nodes"], _ints(c["rows"])
    parents, paths, accepted = st["parent"].tolist(), st["path"].tolist(), st["accepted"].tolist()
    family = torch.zeros((len(rows), T, T), dtype=torch.bool)
    for b, parent in enumerate(parents):
        for t in range(T):
            if parent[t] >= 0:
                family[b, t] = family[b, parent[t]]
            family[b, t, t] = True
    family = family.cuda()
    outs, caches = [], [[], []]
    for q, kn, vn, kc, vc in zip(st["q"], st["kn"], st["vn"], st["kc"], st["vc"]):
        out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
        kc, vc = kc.clone(), vc.clone()
        for b, n in enumerate(rows):
            hidden = torch.cat([torch.zeros((T, n), dtype=torch.bool, device="cuda"), ~family[b]], 1)
            for h in range(c["kv_heads"]):
                kc[b, h, n:n + T], vc[b, h, n:n + T] = kn[b, :, h], vn[b, :, h]
                k64, v64 = kc[b, h, :n + T].double(), vc[b, h, :n + T].double()
                for head in range(h * G, (h + 1) * G):
                    logits = (q[b, :, head].double() @ k64.t() / math.sqrt(c["head_dim"])).masked_fill_(hidden, -math.inf)
                    out[b, :, head] = torch.softmax(logits, -1) @ v64
            for i in range(accepted[b]):
                kc[b, :, n + i], vc[b, :, n + i] = kn[b, paths[b][i]], vn[b, paths[b][i]]
        outs.append(out)
        caches[0].append(kc)
        caches[1].append(vc)
    return [st["first"] + st["accepted"][:, None]] + outs + caches[0] + caches[1]


def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    return {"norm_rope": _exact_norm_rope, "store": _exact_store, "step": _exact_step, "tree": _exact_tree}[case["kind"]](st)
