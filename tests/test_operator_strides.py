"""Strides past any memory: a product of one with the bytes of an element or with the rows of a tile does not fit 64 bits, so that checks and addresses made of it would be of another number.
Refused, through the C ABI with pointers that are never dereferenced, no GPU."""
import ctypes as C

import pytest

import paper_2503_17922_amd as W

NULL, FAKE = C.c_void_p(0), [C.c_void_p((i + 1) << 20) for i in range(8)]


@pytest.mark.parametrize("which", ["q_strides", "kv_strides", "out_strides"])
@pytest.mark.parametrize("axis", [0, 1, 2])
@pytest.mark.parametrize("stride", [1 << 57, 1 << 56, 1 << 62, (1 << 63) - 64])
def test_attention_strides_past_any_memory(which, axis, stride):
    strides = [5 * 128, 128, 128]
    strides[axis] = stride
    shape = W.AttentionShape(q_len=[5, 5], n_q_heads=1, n_kv_heads=1, head_dim=128, dtype=W.WKV_BF16, **{which: tuple(strides)})
    assert W.lib().wkv_attention_workspace_bytes(shape.ref()) == 0 and len(W.lib().wkv_last_error()) > 5
    assert W.lib().wkv_prefill_attention(shape.ref(), *FAKE[:4], NULL, FAKE[4], 1 << 40, NULL) in (W.WKV_ERR_INVALID_ARG, W.WKV_ERR_UNSUPPORTED)


@pytest.mark.parametrize("which", ["q_strides", "k_strides", "q_out_strides", "k_out_strides"])
@pytest.mark.parametrize("stride", [1 << 57, 1 << 62])
def test_rope_strides_past_any_memory(which, stride):
    for axis in range(3):
        strides = [5 * 128, 128, 128]
        strides[axis] = stride
        kw = dict(q_strides=(640, 128, 128), k_strides=(640, 128, 128))
        kw[which] = tuple(strides)
        shape = W.RopeShape(batch=2, n_tokens=5, n_q_heads=1, n_kv_heads=1, head_dim=128, dtype=W.WKV_BF16, inv_freq=[1.0] * 64, **kw)
        assert W.lib().wkv_rope(shape.ref(), *FAKE[:5], NULL) in (W.WKV_ERR_INVALID_ARG, W.WKV_ERR_UNSUPPORTED)


@pytest.mark.parametrize("axis", [0, 1, 2])
@pytest.mark.parametrize("stride", [1 << 57, 1 << 62])
def test_cache_strides_past_any_memory(axis, stride):
    strides = [5 * 128, 128, 128]
    strides[axis] = stride
    shape = W.DecodeShape(batch=2, n_q_heads=1, n_kv_heads=1, head_dim=128, dtype=W.WKV_BF16, capacity=5, cache_strides=tuple(strides))
    caches = (C.c_void_p * 1)(FAKE[0])
    l = W.lib()
    assert l.wkv_decode_weighted_workspace_bytes(shape.ref()) == 0 and l.wkv_evict_workspace_bytes(shape.ref()) == 0
    assert l.wkv_decode_step_weighted(shape.ref(), *FAKE[:7], NULL, NULL, FAKE[7], FAKE[0], 1 << 40, NULL) == W.WKV_ERR_INVALID_ARG
    assert l.wkv_cache_evict(shape.ref(), 1, caches, caches, *FAKE[:4], 0, FAKE[4], 1 << 40, NULL) == W.WKV_ERR_INVALID_ARG
