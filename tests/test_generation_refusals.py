"""What the operators of generation refuse, before anything is launched: through the C ABI with pointers that are never dereferenced, no GPU."""
import ctypes as C
import math
import os
import subprocess

import pytest

import paper_2503_17922_amd as W

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, UNSUPPORTED, WORKSPACE = W.WKV_ERR_INVALID_ARG, W.WKV_ERR_UNSUPPORTED, W.WKV_ERR_WORKSPACE
NULL, FAKE, OTHER, ODD, ODD4 = C.c_void_p(0), C.c_void_p(1 << 20), C.c_void_p(2 << 20), C.c_void_p((1 << 20) + 8), C.c_void_p((1 << 20) + 2)
P = lambda i: C.c_void_p(i << 20)


def arrays(*xs):
    return [(C.c_void_p * 65)(*[x.value or 0] * 65) for x in xs]


# ---- norms with rotary positions

def norm_rope(fields=None, positions=FAKE, qw=P(5), kw=P(6), q_in=FAKE, q_out=OTHER, k_in=FAKE, k_out=P(3), **kwargs):
    base = dict(batch=2, n_tokens=5, n_q_heads=8, n_kv_heads=2, head_dim=128, dtype=W.WKV_BF16, inv_freq=[1.0] * 64)
    base.update(kwargs)
    shape = W.NormRopeShape(**base)
    for name, value in (fields or {}).items():
        setattr(shape.c, name, value)
    return W.lib().wkv_norm_rope(shape.ref(), positions, qw, kw, q_in, q_out, k_in, k_out, NULL)


@pytest.mark.parametrize("kw,status", [
    (dict(batch=0), INVALID), (dict(n_tokens=-1), INVALID), (dict(batch=1 << 13, n_tokens=(1 << 12) + 1), UNSUPPORTED),
    (dict(n_q_heads=-1), INVALID), (dict(n_kv_heads=70000), UNSUPPORTED), (dict(head_dim=96), UNSUPPORTED), (dict(dtype=3), INVALID),
    (dict(inv_freq=[1.0] * 20), UNSUPPORTED), (dict(inv_freq=[]), INVALID), (dict(inv_freq=[1.0] * 72), INVALID),
    (dict(inv_freq=[1.0] * 63 + [math.nan]), INVALID), (dict(amplitude=math.nan), INVALID), (dict(amplitude=1e39), INVALID),
    (dict(fields=dict(flags=2)), INVALID), (dict(fields=dict(inv_freq=None)), INVALID), (dict(n_axes=0), INVALID), (dict(n_axes=5), INVALID),
    (dict(n_axes=2, axis_of_pair=[0] * 63 + [2]), INVALID), (dict(n_axes=2, axis_of_pair=[-1] + [0] * 63), INVALID), (dict(axis_of_pair=[0] * 63 + [1]), INVALID),
    (dict(eps=-1e-6), INVALID), (dict(eps=math.nan), INVALID), (dict(eps=math.inf), INVALID),
    (dict(q_strides=(640, 128, 100)), INVALID), (dict(k_out_strides=(640, 128, 132)), INVALID), (dict(q_strides=(-640, 128, 128)), INVALID),
    (dict(k_strides=(640, 64, 128)), INVALID), (dict(q_out_strides=(0, 128, 1 << 50)), INVALID),
    (dict(positions=NULL), INVALID), (dict(positions=ODD4), INVALID), (dict(q_in=NULL), INVALID), (dict(k_out=NULL), INVALID), (dict(q_out=ODD), INVALID),
    (dict(k_in=ODD), INVALID), (dict(qw=ODD), INVALID), (dict(kw=ODD), INVALID), (dict(q_out=FAKE, q_out_strides=(8 * 6 * 128, 6 * 128, 128)), INVALID),
    (dict(q_out=OTHER, k_out=OTHER), INVALID),
])
def test_norm_rope(kw, status):
    assert norm_rope(**kw) == status
    assert len(W.lib().wkv_last_error()) > 5


def test_norm_rope_with_nothing_to_do():
    assert norm_rope(n_tokens=0, positions=NULL, q_in=NULL) == W.WKV_OK
    assert norm_rope(n_q_heads=0, n_kv_heads=0, positions=NULL) == W.WKV_OK
    assert W.lib().wkv_norm_rope(None, *[FAKE] * 7, NULL) == INVALID
    with pytest.raises(ValueError):
        W.NormRopeShape(batch=1, n_tokens=1, n_q_heads=1, n_kv_heads=1, head_dim=64, dtype=W.WKV_F32, inv_freq=[1.0] * 32, n_axes=2, axis_of_pair=[0] * 31)


# ---- caches in 8 and 4 bits

def quantized(fields=None, **kw):
    base = dict(batch=2, n_q_heads=32, n_kv_heads=8, head_dim=128, dtype=W.WKV_BF16, format=W.WKV_CACHE_E4M3, capacity=500, n_rows=100)
    base.update(kw)
    shape = W.QuantizedShape(**base)
    for name, value in (fields or {}).items():
        setattr(shape.c, name, value)
    return shape


BAD_SHAPES = [(dict(batch=0), INVALID), (dict(n_q_heads=30), INVALID), (dict(n_q_heads=72), UNSUPPORTED), (dict(head_dim=32), UNSUPPORTED),
              (dict(capacity=0), INVALID), (dict(capacity=(1 << 30) + 1), UNSUPPORTED), (dict(dtype=-1), INVALID), (dict(flags=2), INVALID),
              (dict(format=2), INVALID), (dict(format=-1), INVALID), (dict(batch=9000), UNSUPPORTED), (dict(scale=-1.0), INVALID), (dict(scale=math.nan), INVALID),
              (dict(code_strides=(0, 128, 120)), INVALID), (dict(code_strides=(0, 112, 128)), INVALID), (dict(code_strides=(-16, 128, 128)), INVALID),
              (dict(code_strides=(0, 64, 128)), INVALID), (dict(code_strides=(0, 128, 64)), INVALID), (dict(code_strides=(0, 128, 1 << 27)), UNSUPPORTED),
              (dict(code_strides=(1 << 50, 128, 128)), INVALID), (dict(format=W.WKV_CACHE_E2M1, code_strides=(0, 64, 48)), INVALID)]


@pytest.mark.parametrize("kw,status", BAD_SHAPES)
def test_quantized_shapes(kw, status):
    sh, lib = quantized(**kw), W.lib()
    assert lib.wkv_decode_quantized_workspace_bytes(sh.ref()) == 0
    assert lib.wkv_decode_step_quantized(sh.ref(), *[FAKE] * 10, 1 << 40, NULL) == status
    a = arrays(FAKE)[0]
    assert lib.wkv_cache_quantize(sh.ref(), 1, a, a, NULL, NULL, NULL, a, a, a, a, NULL) == status
    assert lib.wkv_cache_dequantize(sh.ref(), 1, a, a, a, a, NULL, NULL, a, a, NULL) == status
    assert len(lib.wkv_last_error()) > 5


def test_quantized_step_arguments():
    sh, lib = quantized(), W.lib()
    need = lib.wkv_decode_quantized_workspace_bytes(sh.ref())
    assert need >= 2 * 8 * 4 * 130 * 4

    def call(change, nbytes=need):
        a = [FAKE] * 10
        for i, x in change.items():
            a[i] = x
        return lib.wkv_decode_step_quantized(sh.ref(), *a, nbytes, NULL)

    for i in range(9):
        assert call({i: NULL}) == INVALID, i
    for i in (0, 1, 2, 3, 5):
        assert call({i: ODD}) == INVALID, i
    for i in (4, 6, 7, 8):
        assert call({i: ODD4}) == INVALID, i
    assert call({9: NULL}) == WORKSPACE and call({9: ODD}) == WORKSPACE and call({}, need - 1) == WORKSPACE


@pytest.mark.parametrize("fields,status", [
    (dict(n_rows=-1), INVALID), (dict(n_rows=1 << 27), UNSUPPORTED), (dict(row_stride_t=100), INVALID), (dict(row_stride_h=64), INVALID),
    (dict(row_stride_b=-128), INVALID), (dict(row_stride_t=1 << 50), INVALID)])
def test_rows_of_plain_tensors(fields, status):
    sh, lib, a = quantized(fields), W.lib(), arrays(FAKE)[0]
    assert lib.wkv_cache_quantize(sh.ref(), 1, a, a, FAKE, NULL, NULL, a, a, a, a, NULL) == status
    assert lib.wkv_cache_dequantize(sh.ref(), 1, a, a, a, a, NULL, NULL, a, a, NULL) == status


def test_row_arguments():
    sh, lib = quantized(), W.lib()
    ok, bad, odd, odd4 = arrays(FAKE, NULL, ODD, ODD4)

    def put(n=2, layers=(ok,) * 6, tok=FAKE, keep=FAKE, first=FAKE, shape=sh):
        return lib.wkv_cache_quantize(shape.ref(), n, layers[0], layers[1], tok, keep, first, *layers[2:], NULL)

    def get(n=2, layers=(ok,) * 6, first=FAKE, valid=FAKE, shape=sh):
        return lib.wkv_cache_dequantize(shape.ref(), n, *layers[2:], first, valid, layers[0], layers[1], NULL)

    for call in (put, get):
        assert call(n=0) == INVALID and call(n=65) == INVALID
        for i in range(6):
            assert call(layers=tuple(None if j == i else ok for j in range(6))) == INVALID
            assert call(layers=tuple(bad if j == i else ok for j in range(6))) == INVALID
            wrong = odd4 if i in (3, 5) else odd
            assert call(layers=tuple(wrong if j == i else ok for j in range(6))) == INVALID
    assert put(tok=ODD4) == INVALID and put(keep=ODD4) == INVALID and put(first=ODD4) == INVALID and get(first=ODD4) == INVALID and get(valid=ODD4) == INVALID
    few = quantized(dict(row_capacity=99))
    assert put(shape=few, tok=NULL) == INVALID and put(shape=quantized(dict(row_capacity=-1))) == INVALID
    none = quantized(dict(n_rows=0))
    assert put(shape=none) == W.WKV_OK and get(shape=none) == W.WKV_OK


# ---- trees of drafted tokens

def tree(fields=None, **kw):
    base = dict(batch=2, n_q_heads=32, n_kv_heads=8, head_dim=128, dtype=W.WKV_BF16, n_nodes=16, capacity=500)
    base.update(kw)
    shape = W.TreeShape(**base)
    for name, value in (fields or {}).items():
        setattr(shape.c, name, value)
    return shape


@pytest.mark.parametrize("kw,status", [
    (dict(batch=0), INVALID), (dict(n_q_heads=30), INVALID), (dict(n_kv_heads=0), INVALID), (dict(n_q_heads=72), UNSUPPORTED), (dict(head_dim=32), UNSUPPORTED),
    (dict(n_nodes=0), INVALID), (dict(n_nodes=65), UNSUPPORTED), (dict(capacity=0), INVALID), (dict(capacity=(1 << 30) + 1), UNSUPPORTED), (dict(dtype=-1), INVALID),
    (dict(flags=2), INVALID), (dict(batch=9000), UNSUPPORTED), (dict(scale=-1.0), INVALID), (dict(scale=math.inf), INVALID),
    (dict(cache_strides=(8, 8, 8)), INVALID), (dict(cache_strides=(0, 128, 1 << 24)), UNSUPPORTED), (dict(q_strides=(0, 128, 100)), INVALID),
    (dict(new_strides=(0, 64, 128)), INVALID), (dict(new_strides=(0, 128, 1 << 24)), UNSUPPORTED), (dict(out_strides=(0, 128, 1 << 50)), INVALID)])
def test_tree_shapes(kw, status):
    sh, lib = tree(**kw), W.lib()
    assert lib.wkv_tree_workspace_bytes(sh.ref()) == 0
    assert lib.wkv_decode_tree(sh.ref(), *[P(i + 1) for i in range(8)], FAKE, 1 << 40, NULL) == status
    a = arrays(FAKE)[0]
    assert lib.wkv_tree_accept(sh.ref(), 1, a, a, FAKE, FAKE, FAKE, NULL) == status
    assert len(lib.wkv_last_error()) > 5


def test_tree_arguments():
    sh, lib = tree(), W.lib()
    need = lib.wkv_tree_workspace_bytes(sh.ref())
    assert need > 0 and need % 256 == 0

    def call(change, nbytes=need):
        a = [P(i + 1) for i in range(8)] + [FAKE]
        for i, x in change.items():
            a[i] = x
        return lib.wkv_decode_tree(sh.ref(), *a, nbytes, NULL)

    for i in range(8):
        assert call({i: NULL}) == INVALID, i
    for i in (0, 1, 2, 4, 5, 7):
        assert call({i: ODD}) == INVALID, i
    for i in (3, 6):
        assert call({i: ODD4}) == INVALID, i
    for i in (0, 1, 2, 4, 5):
        assert call({7: P(i + 1)}) == INVALID                # out in the memory of an input
    assert call({8: NULL}) == WORKSPACE and call({8: ODD}) == WORKSPACE and call({}, need - 1) == WORKSPACE


def test_acceptance_arguments():
    sh, lib = tree(), W.lib()
    ok, bad, odd = arrays(FAKE, NULL, ODD)

    def call(n=2, k=ok, v=ok, small=(FAKE,) * 3):
        return lib.wkv_tree_accept(sh.ref(), n, k, v, *small, NULL)

    assert call(n=0) == INVALID and call(n=65) == INVALID and call(k=None) == INVALID and call(v=None) == INVALID and call(v=bad) == INVALID and call(k=odd) == INVALID
    for i in range(3):
        assert call(small=tuple(NULL if j == i else FAKE for j in range(3))) == INVALID
        assert call(small=tuple(ODD4 if j == i else FAKE for j in range(3))) == INVALID


# ---- the binding

CALLS = {
    "norm_rope": (lambda s, x: W.wkv_norm_rope(s, x, x, x, x, x, x, x, stream=0),
                  lambda: W.NormRopeShape(batch=1, n_tokens=1, n_q_heads=1, n_kv_heads=1, head_dim=64, dtype=W.WKV_F32, inv_freq=[1.0] * 32)),
    "quantize": (lambda s, x: W.wkv_cache_quantize(s, [x], [x], x, x, x, [x], [x], [x], [x], stream=0), quantized),
    "dequantize": (lambda s, x: W.wkv_cache_dequantize(s, [x], [x], [x], [x], x, x, [x], [x], stream=0), quantized),
    "step": (lambda s, x: W.wkv_decode_step_quantized(s, *[x] * 10, stream=0), quantized),
    "tree": (lambda s, x: W.wkv_decode_tree(s, *[x] * 9, stream=0), tree),
    "accept": (lambda s, x: W.wkv_tree_accept(s, [x], [x], x, x, x, stream=0), tree),
}


@pytest.mark.parametrize("name", list(CALLS))
def test_the_binding(name):
    import torch
    call, shape = CALLS[name]
    with pytest.raises(W.WkvError, match="NULL"):
        call(shape(), None)
    with pytest.raises(ValueError, match="GPU memory"):
        call(shape(), torch.zeros(16))
    for _, other in CALLS.values():
        if type(other()) is not type(shape()):
            with pytest.raises(C.ArgumentError):
                call(other(), None)
    with pytest.raises(AttributeError):
        call(None, None)


def test_sequences_of_different_lengths():
    with pytest.raises(ValueError, match="layers"):
        W.wkv_cache_quantize(quantized(), [None], [None, None], None, None, None, [None], [None], [None], [None], stream=0)
    with pytest.raises(ValueError, match="layers"):
        W.wkv_cache_dequantize(quantized(), [None], [None], [None], [None], None, None, [None], [], stream=0)
    with pytest.raises(ValueError, match="layers"):
        W.wkv_tree_accept(tree(), [None], [None, None], None, None, None, stream=0)
    with pytest.raises(W.WkvError, match="n_layers"):
        W.wkv_tree_accept(tree(), [None] * 70, [None] * 70, None, None, None, stream=0)


def test_host_side_under_sanitizers(tmp_path):
    """Validation and launch plans, built for the CPU with ASan + UBSan and driven over a sweep of shapes
    (tests/c/generation_validation.cpp); the launchers are stand-ins that check what they are given."""
    from paper_2503_17922_amd import build as B
    exe = B.build_host_sanitized(str(tmp_path), [os.path.join(B.CSRC, "wkv_operators.cpp"), os.path.join(B.CSRC, "wkv_generation.cpp"),
                                                 os.path.join(ROOT, "tests", "c", "generation_validation.cpp"),
                                                 os.path.join(ROOT, "tests", "c", "launch_stubs.cpp")], "generation_validation")
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0", UBSAN_OPTIONS="print_stacktrace=1")
    env.pop("LD_PRELOAD", None)
    res = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
    assert res.returncode == 0, res.stdout[-2000:] + res.stderr[-4000:]
    assert res.stdout.strip().endswith("ok (0 checks failed)")
