"""wkv_cache_quantize and wkv_cache_dequantize of as many rows as they take, more than one launch's grid holds."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2503_17922_amd as W
from tests import few_bits as F

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,n", [(128, 1 << 30), (64, 1 << 30), (128, (1 << 27) + 33), (64, (1 << 28) + 1)])
def test_rows_behind_the_first_launch(device, d, n):
    # the cache and the plain rows hold the call's last 100 rows; all other rows fall outside of both
    cap, dtype, fmt = 100, W.WKV_BF16, W.WKV_CACHE_E4M3
    g = torch.Generator(device=device).manual_seed(50)
    x = torch.randn((2, cap, d), device=device, generator=g).bfloat16()
    first = torch.tensor([[cap - n]], dtype=torch.int32, device=device)
    tok = torch.full((n,), -1, dtype=torch.int32, device=device)
    tok[n - cap:] = torch.randperm(cap, device=device, generator=g).to(torch.int32)
    codes = [torch.full((1, 1, cap, d), 0xee, dtype=torch.uint8, device=device) for _ in range(2)]
    scales = [torch.full((1, 1, cap, d // 32), 0xee, dtype=torch.uint8, device=device) for _ in range(2)]
    into = W.QuantizedShape(batch=1, n_kv_heads=1, head_dim=d, dtype=dtype, format=fmt, capacity=cap, n_rows=n, row_capacity=cap, row_strides=(0, cap * d, d))
    W.wkv_cache_quantize(into, [x[0]], [x[1]], tok, None, first, [codes[0]], [scales[0]], [codes[1]], [scales[1]])
    torch.cuda.synchronize()
    for i in range(2):
        c, s = F.encode(x[i, tok[n - cap:].long()], fmt)
        assert np.array_equal(codes[i][0, 0].cpu().numpy(), c) and np.array_equal(scales[i][0, 0].cpu().numpy(), s)
    del tok
    # and back: the rows that the cache does not hold are not touched, so that the last 100 rows of the outputs are all there is of them
    out = torch.full((2, cap + 2, d), 7.0, dtype=torch.bfloat16, device=device)
    back = W.QuantizedShape(batch=1, n_kv_heads=1, head_dim=d, dtype=dtype, format=fmt, capacity=cap, n_rows=n, row_capacity=n, row_strides=(0, n * d, d))
    one = lambda p: (C.c_void_p * 1)(p)
    starts = [out[i, 1].data_ptr() - (n - cap) * d * 2 for i in range(2)]
    assert W.lib().wkv_cache_dequantize(back.ref(), 1, one(codes[0].data_ptr()), one(scales[0].data_ptr()), one(codes[1].data_ptr()), one(scales[1].data_ptr()),
                                        C.c_void_p(first.data_ptr()), None, one(starts[0]), one(starts[1]), C.c_void_p(torch.cuda.current_stream().cuda_stream)) == W.WKV_OK
    torch.cuda.synchronize()
    for i in range(2):
        assert torch.equal(out[i, 1:-1].double(), F.decode_torch(codes[i][0, 0], scales[i][0, 0], fmt))
        assert (out[i, 0] == 7.0).all() and (out[i, -1] == 7.0).all()
