"""What the operators around the compression refuse, before anything is launched: through the C ABI with pointers that are never
dereferenced, no GPU.  Derived sizes and frequencies likewise."""
import ctypes as C
import math
import os
import subprocess

import pytest

import paper_2503_17922_amd as W

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, UNSUPPORTED, WORKSPACE = W.WKV_ERR_INVALID_ARG, W.WKV_ERR_UNSUPPORTED, W.WKV_ERR_WORKSPACE
NULL, FAKE, OTHER, ODD = C.c_void_p(0), C.c_void_p(1 << 20), C.c_void_p(2 << 20), C.c_void_p((1 << 20) + 8)


def rope(fields=None, positions=FAKE, q_in=FAKE, q_out=OTHER, k_in=FAKE, k_out=C.c_void_p(3 << 20), **kw):
    base = dict(batch=2, n_tokens=5, n_q_heads=8, n_kv_heads=2, head_dim=128, dtype=W.WKV_BF16, inv_freq=[1.0] * 64)
    base.update(kw)
    shape = W.RopeShape(**base)
    for name, value in (fields or {}).items():
        setattr(shape.c, name, value)
    return W.lib().wkv_rope(shape.ref(), positions, q_in, q_out, k_in, k_out, NULL)


@pytest.mark.parametrize("kw,status", [
    (dict(batch=0), INVALID), (dict(n_tokens=-1), INVALID), (dict(batch=1 << 13, n_tokens=(1 << 12) + 1), UNSUPPORTED),
    (dict(n_q_heads=-1), INVALID), (dict(n_kv_heads=70000), UNSUPPORTED), (dict(head_dim=96), UNSUPPORTED), (dict(dtype=3), INVALID),
    (dict(inv_freq=[1.0] * 20), UNSUPPORTED), (dict(inv_freq=[]), INVALID), (dict(inv_freq=[1.0] * 72), INVALID),
    (dict(inv_freq=[1.0] * 63 + [math.nan]), INVALID), (dict(inv_freq=[math.inf] * 64), INVALID), (dict(amplitude=math.nan), INVALID),
    (dict(amplitude=1e39), INVALID), (dict(fields=dict(flags=4)), INVALID), (dict(fields=dict(inv_freq=None)), INVALID),
    (dict(q_strides=(640, 128, 100)), INVALID), (dict(k_out_strides=(640, 128, 132)), INVALID), (dict(q_strides=(-640, 128, 128)), INVALID),
    (dict(k_strides=(640, 64, 128)), INVALID),
    (dict(positions=NULL), INVALID), (dict(positions=C.c_void_p(4098)), INVALID), (dict(q_in=NULL), INVALID), (dict(k_out=NULL), INVALID),
    (dict(q_out=ODD), INVALID), (dict(k_in=ODD), INVALID), (dict(q_out=FAKE, q_out_strides=(8 * 6 * 128, 6 * 128, 128)), INVALID),
    (dict(q_out=OTHER, k_out=OTHER), INVALID),
])
def test_rope(kw, status):
    assert rope(**kw) == status
    assert len(W.lib().wkv_last_error()) > 5


def test_rope_with_nothing_to_do():
    assert rope(n_tokens=0, positions=NULL, q_in=NULL) == W.WKV_OK
    assert rope(n_q_heads=0, n_kv_heads=0, positions=NULL) == W.WKV_OK
    assert W.lib().wkv_rope(None, FAKE, FAKE, FAKE, FAKE, FAKE, NULL) == INVALID


@pytest.mark.parametrize("args", [
    (0, 1e4, 0, 1.0, 0), (7, 1e4, 0, 1.0, 0), (1 << 17, 1e4, 0, 1.0, 0), (128, 1.0, 0, 1.0, 0), (128, math.nan, 0, 1.0, 0), (128, math.inf, 0, 1.0, 0),
    (128, 1e4, 5, 1.0, 0), (128, 1e4, -1, 1.0, 0), (128, 1e4, W.WKV_ROPE_LINEAR, 0.5, 0), (128, 1e4, W.WKV_ROPE_BASE, math.nan, 0),
    (128, 1e4, W.WKV_ROPE_PARTS, 4.0, 0), (128, 1e4, W.WKV_ROPE_WAVELENGTH, 4.0, -5), (2, 1e4, W.WKV_ROPE_BASE, 2.0, 0),
])
def test_rope_frequencies_refusals(args):
    with pytest.raises(W.WkvError) as e:
        W.wkv_rope_frequencies(*args)
    assert e.value.status == INVALID


def test_rope_frequencies():
    r, theta = 128, 500000.0
    plain, one = W.wkv_rope_frequencies(r, theta)
    assert one == 1.0 and plain[0] == 1.0
    for i, f in enumerate(plain):
        assert f == pytest.approx(theta ** (-2.0 * i / r), rel=1e-14)
    linear, _ = W.wkv_rope_frequencies(r, theta, W.WKV_ROPE_LINEAR, 4.0)
    assert linear == pytest.approx([f / 4 for f in plain], rel=1e-14)
    base, _ = W.wkv_rope_frequencies(r, theta, W.WKV_ROPE_BASE, 4.0)
    assert base[0] == 1.0 and base[-1] == pytest.approx(plain[-1] / 4, rel=1e-12)
    assert all(x > y for x, y in zip(base, base[1:]))
    for kind in (W.WKV_ROPE_PARTS, W.WKV_ROPE_WAVELENGTH):
        got, amplitude = W.wkv_rope_frequencies(r, theta, kind, 8.0, 8192)
        turns = [8192 * f / (2 * math.pi) for f in plain]
        low, high = (1.0, 32.0) if kind == W.WKV_ROPE_PARTS else (1.0, 4.0)
        channel = lambda n: r * math.log(8192 / (n * 2 * math.pi)) / (2 * math.log(theta))
        for i, (f, g, n) in enumerate(zip(plain, got, turns)):
            if n >= high * (1.5 if kind == W.WKV_ROPE_PARTS else 1.0):      # (by whole channels there)
                assert g == f
            elif n <= low / (1.5 if kind == W.WKV_ROPE_PARTS else 1.0):
                assert g == pytest.approx(f / 8, rel=1e-14)
            else:
                assert f / 8 <= g <= f
                lo, hi = math.floor(channel(32.0)), math.ceil(channel(1.0))
                share = 1 - min(max((i - lo) / (hi - lo), 0), 1) if kind == W.WKV_ROPE_PARTS else (n - 1) / 3
                assert g == pytest.approx(f * share + f / 8 * (1 - share), rel=1e-12)
        assert amplitude == pytest.approx(0.1 * math.log(8.0) + 1 if kind == W.WKV_ROPE_PARTS else 1.0, rel=1e-15)
    # a context in which every channel turns less than once: all but the first slow by the whole factor
    tiny, _ = W.wkv_rope_frequencies(r, theta, W.WKV_ROPE_PARTS, 8.0, 1)
    assert tiny[1:] == pytest.approx([f / 8 for f in plain[1:]], rel=1e-14)


def attention(fields=None, q=FAKE, k=OTHER, v=C.c_void_p(3 << 20), out=C.c_void_p(4 << 20), lse=FAKE, ws=FAKE, nbytes=1 << 40, **kw):
    base = dict(q_len=[100, 5], n_q_heads=8, n_kv_heads=2, head_dim=128, dtype=W.WKV_BF16, lse_rows=4)
    base.update(kw)
    shape = W.AttentionShape(**base)
    for name, value in (fields or {}).items():
        setattr(shape.c, name, value)
    st = W.lib().wkv_prefill_attention(shape.ref(), q, k, v, out, lse, ws, nbytes, NULL)
    return st, shape


SHAPES = [
    (dict(q_len=[]), INVALID), (dict(q_len=[1] * 65), UNSUPPORTED), (dict(n_q_heads=9), INVALID), (dict(n_kv_heads=0), INVALID), (dict(dtype=9), INVALID),
    (dict(head_dim=80), UNSUPPORTED), (dict(scale=-1.0), INVALID), (dict(scale=math.nan), INVALID), (dict(scale=math.inf), INVALID),
    (dict(lse_rows=-1), INVALID), (dict(lse_rows=(1 << 28) + 1), UNSUPPORTED), (dict(flags=1), INVALID), (dict(q_len=[-1, 5]), INVALID), (dict(k_len=[3, -2]), INVALID),
    (dict(q_start=[0, -1]), INVALID), (dict(k_start=[-7, 0]), INVALID), (dict(q_strides=(0, 128, 100)), INVALID), (dict(kv_strides=(0, 64, 128)), INVALID),
    (dict(out_strides=(0, 128, 132)), INVALID), (dict(kv_strides=(0, 128, 1 << 25)), UNSUPPORTED), (dict(q_len=[2 ** 31 - 1, 1], q_strides=(0, 128, 128)), UNSUPPORTED),
    (dict(q_len=[1, 1], k_len=[2 ** 31 - 1, 1], kv_strides=(0, 128, 128)), UNSUPPORTED),
    (dict(q_len=[1 << 20] * 64, n_q_heads=64, n_kv_heads=64, q_strides=(0, 128, 128), kv_strides=(0, 128, 128)), UNSUPPORTED), (dict(fields=dict(q_len=None)), INVALID),
]


@pytest.mark.parametrize("kw,status", SHAPES)
def test_attention_shapes(kw, status):
    st, shape = attention(**kw)
    assert st == status and len(W.lib().wkv_last_error()) > 5
    assert W.lib().wkv_attention_workspace_bytes(shape.ref()) == 0


@pytest.mark.parametrize("kw,status", [
    (dict(q=NULL), INVALID), (dict(k=NULL), INVALID), (dict(v=NULL), INVALID), (dict(out=NULL), INVALID), (dict(q=ODD), INVALID), (dict(out=ODD), INVALID),
    (dict(lse=NULL), INVALID), (dict(lse=C.c_void_p(4098)), INVALID), (dict(out=FAKE), INVALID), (dict(out=OTHER), INVALID),
    (dict(ws=NULL), WORKSPACE), (dict(ws=C.c_void_p(4096 + 64)), WORKSPACE), (dict(nbytes=10), WORKSPACE),
])
def test_attention_arguments(kw, status):
    assert attention(**kw)[0] == status


def test_attention_with_nothing_to_do():
    assert attention(q_len=[0, 0], lse_rows=0, lse=NULL)[0] == W.WKV_OK
    assert attention(q_len=[0], k_len=[100], lse_rows=0, lse=NULL)[0] == W.WKV_OK
    assert W.lib().wkv_attention_workspace_bytes(None) == 0
    with pytest.raises(ValueError):
        W.AttentionShape(q_len=[1, 2], k_len=[3], n_q_heads=1, n_kv_heads=1, head_dim=64, dtype=W.WKV_F32)


def decode_shape(**kw):
    base = dict(batch=2, n_q_heads=32, n_kv_heads=8, head_dim=128, dtype=W.WKV_BF16, capacity=500)
    base.update(kw)
    return W.DecodeShape(**base)


BAD_CACHES = [(dict(batch=0), INVALID), (dict(n_q_heads=30), INVALID), (dict(n_q_heads=72), UNSUPPORTED), (dict(head_dim=32), UNSUPPORTED),
              (dict(capacity=0), INVALID), (dict(capacity=(1 << 30) + 1), UNSUPPORTED), (dict(dtype=-1), INVALID), (dict(flags=2), INVALID),
              (dict(cache_strides=(8, 8, 8)), INVALID), (dict(batch=9000), UNSUPPORTED)]


@pytest.mark.parametrize("kw,status", BAD_CACHES)
def test_cache_shapes(kw, status):
    sh, lib = decode_shape(**kw), W.lib()
    assert lib.wkv_decode_weighted_workspace_bytes(sh.ref()) == 0 and lib.wkv_evict_workspace_bytes(sh.ref()) == 0
    assert lib.wkv_decode_step_weighted(sh.ref(), *[FAKE] * 11, 1 << 40, NULL) == status
    arr = (C.c_void_p * 1)(FAKE.value)
    assert lib.wkv_cache_evict(sh.ref(), 1, arr, arr, FAKE, FAKE, FAKE, FAKE, 0, FAKE, 1 << 40, NULL) == status


def test_weighted_step_arguments():
    sh, lib = decode_shape(), W.lib()
    need = lib.wkv_decode_weighted_workspace_bytes(sh.ref())
    assert need > lib.wkv_decode_workspace_bytes(sh.ref()) + 2 * 32 * 500 * 4

    def call(change, nbytes=need):
        a = [FAKE] * 11
        for i, x in change.items():
            a[i] = x
        return lib.wkv_decode_step_weighted(sh.ref(), *a, nbytes, NULL)

    for i in range(7):
        assert call({i: NULL}) == INVALID, i
    assert call({9: NULL}) == INVALID and call({10: NULL}) == WORKSPACE
    assert call({7: NULL}) == INVALID and call({8: NULL}) == INVALID            # positions and their array go together
    for i in range(5):
        assert call({i: ODD}) == INVALID
    for i in (5, 6, 7, 8, 9):
        assert call({i: C.c_void_p(4097)}) == INVALID
    assert call({10: ODD}) == WORKSPACE and call({}, need - 1) == WORKSPACE


def test_eviction_arguments():
    sh, lib = decode_shape(), W.lib()
    need = lib.wkv_evict_workspace_bytes(sh.ref())
    assert need >= 2 * 8 * (4 + 250 * 8)
    ok, bad, odd = ((C.c_void_p * 64)(*[x] * 64) for x in (FAKE.value, 0, ODD.value))

    def call(n=2, k=ok, v=ok, small=(FAKE,) * 4, recent=0, ws=FAKE, nbytes=need):
        return lib.wkv_cache_evict(sh.ref(), n, k, v, *small, recent, ws, nbytes, NULL)

    assert call(n=0) == INVALID and call(n=65) == INVALID and call(k=None) == INVALID and call(v=bad) == INVALID and call(k=odd) == INVALID
    for i in range(4):
        assert call(small=tuple(NULL if j == i else FAKE for j in range(4))) == INVALID
        assert call(small=tuple(C.c_void_p(4098) if j == i else FAKE for j in range(4))) == INVALID
    assert call(recent=-1) == INVALID and call(ws=NULL) == WORKSPACE and call(ws=ODD) == WORKSPACE and call(nbytes=need - 1) == WORKSPACE


def test_the_binding_refuses_what_is_not_on_the_gpu():
    import torch
    x = torch.zeros(16)
    sh = decode_shape()
    with pytest.raises(ValueError, match="GPU memory"):
        W.wkv_decode_step_weighted(sh, x, x, x, x, x, x, x, x, x, x, x, stream=0)
    with pytest.raises(ValueError, match="GPU memory"):
        W.wkv_cache_evict(sh, [x], [x], x, x, x, x, 0, x, stream=0)
    with pytest.raises(ValueError, match="GPU memory"):
        W.wkv_prefill_attention(W.AttentionShape(q_len=[1], n_q_heads=1, n_kv_heads=1, head_dim=64, dtype=W.WKV_F32), x, x, x, x, None, x, stream=0)
    with pytest.raises(ValueError, match="GPU memory"):
        W.wkv_rope(W.RopeShape(batch=1, n_tokens=1, n_q_heads=1, n_kv_heads=0, head_dim=64, dtype=W.WKV_F32, inv_freq=[1.0] * 32), x, x, x, None, None, stream=0)


RIGHT = {
    "rope": (lambda s: W.wkv_rope(s, None, None, None, None, None, stream=0),
             lambda: W.RopeShape(batch=1, n_tokens=1, n_q_heads=1, n_kv_heads=1, head_dim=64, dtype=W.WKV_F32, inv_freq=[1.0] * 32)),
    "prefill": (lambda s: W.wkv_prefill_attention(s, None, None, None, None, None, None, stream=0),
                lambda: W.AttentionShape(q_len=[1], n_q_heads=1, n_kv_heads=1, head_dim=64, dtype=W.WKV_F32)),
    "weighted": (lambda s: W.wkv_decode_step_weighted(s, *[None] * 11, stream=0), decode_shape),
    "evict": (lambda s: W.wkv_cache_evict(s, [None], [None], None, None, None, None, 0, None, stream=0), decode_shape),
}


@pytest.mark.parametrize("name", list(RIGHT))
def test_another_structure_is_refused(name):
    call, right = RIGHT[name]
    with pytest.raises(W.WkvError, match="NULL"):
        call(right())
    for other in ("rope", "prefill", "weighted"):
        wrong = RIGHT[other][1]()
        if type(wrong) is not type(right()):
            with pytest.raises(C.ArgumentError):
                call(wrong)
    with pytest.raises(AttributeError):
        call(None)


def test_host_side_under_sanitizers(tmp_path):
    """Validation and launch plans of these operators, built for the CPU with ASan + UBSan and driven over a sweep of
    shapes (tests/c/operators_validation.cpp); the launchers are stand-ins that check what they are given."""
    from paper_2503_17922_amd import build as B
    exe = B.build_host_sanitized(str(tmp_path), [os.path.join(B.CSRC, "wkv_operators.cpp"), os.path.join(ROOT, "tests", "c", "operators_validation.cpp"),
                                                 os.path.join(ROOT, "tests", "c", "launch_stubs.cpp")], "operators_validation")
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0", UBSAN_OPTIONS="print_stacktrace=1")
    env.pop("LD_PRELOAD", None)
    res = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
    assert res.returncode == 0, res.stdout[-2000:] + res.stderr[-4000:]
    assert res.stdout.strip().endswith("ok (0 checks failed)")
