"""wkv_prefill_attention where there is nothing to read: tensors without elements have no address, which is no error."""
import ctypes as C

import pytest
import torch

import paper_2503_17922_amd as W

NULL, FAKE = C.c_void_p(0), [C.c_void_p((i + 1) << 20) for i in range(8)]
INVALID = W.WKV_ERR_INVALID_ARG


def call(q_len, k_len, q, k, v, out, lse_rows=0):
    shape = W.AttentionShape(q_len=q_len, k_len=k_len, n_q_heads=2, n_kv_heads=1, head_dim=64, dtype=W.WKV_BF16, lse_rows=lse_rows)
    return W.lib().wkv_prefill_attention(shape.ref(), q, k, v, out, NULL, FAKE[4], 1 << 30, NULL)


def test_nothing_at_all():
    assert call([0, 0], [0, 0], NULL, NULL, NULL, NULL) == W.WKV_OK
    assert call([0, 0], [5, 0], NULL, FAKE[1], FAKE[2], NULL) == W.WKV_OK


@pytest.mark.parametrize("q_len,k_len,q,k,v,out", [([0, 3], [0, 3], NULL, *FAKE[1:4]), ([3, 0], [0, 3], *FAKE[:3], NULL), ([3, 1], [0, 1], FAKE[0], NULL, *FAKE[2:4]),
                                                   ([3, 1], [0, 1], *FAKE[:2], NULL, FAKE[3])])
def test_what_is_read_or_written_has_an_address(q_len, k_len, q, k, v, out):
    assert call(q_len, k_len, q, k, v, out) == INVALID


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_rows_without_any_keys(device, dtype):
    q, out = torch.randn((2, 4, 150, 64), device=device).to(dtype), torch.ones((2, 4, 150, 64), device=device, dtype=dtype)
    k = torch.empty((2, 2, 0, 64), device=device, dtype=dtype)
    lse = torch.zeros((2, 4, 160), device=device)
    number = {torch.float32: W.WKV_F32, torch.bfloat16: W.WKV_BF16, torch.float16: W.WKV_F16}[dtype]
    kw = dict(n_q_heads=4, n_kv_heads=2, head_dim=64, dtype=number)
    ws = torch.empty(256, device=device, dtype=torch.uint8)
    W.wkv_prefill_attention(W.AttentionShape(q_len=[150, 7], k_len=[0, 0], lse_rows=160, **kw), q, k, k, out, lse, ws)
    assert (out[0] == 0).all() and (out[1, :, :7] == 0).all() and (out[1, :, 7:] == 1).all() and (lse == -float("inf")).all()
    # no rows either, normalisers of them all the same
    lse.zero_()
    W.wkv_prefill_attention(W.AttentionShape(q_len=[0, 0], k_len=[0, 0], lse_rows=160, **kw), k, k, k, k, lse, ws)
    assert (lse == -float("inf")).all()
