"""wkv_norm_rope without an eps, or next to none, on rows whose squares leave fp32's normal numbers: a row's own size goes out of the result all the same."""
import pytest
import torch

import paper_2503_17922_amd as W
from tests.test_gpu_norm_rope import TYPES, check, expected, weights

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("interleaved,axes", [(False, 1), (True, 3)])
@pytest.mark.parametrize("eps", [0.0, 1e-44, 1e-38, 7e-31, 9e-31, 1e-25])
def test_rows_near_the_smallest_numbers(device, dtype, d, interleaved, axes, eps):
    inv, _ = W.wkv_rope_frequencies(d, 10000.0)
    g = torch.Generator(device=device).manual_seed(40)
    # in fp16 the smallest numbers are 6e-8; in the others 1e-45 and 9e-41
    sizes = [2.0 ** -24 * 3, 1e-5, 1.0] if dtype == W.WKV_F16 else [3e-39, 1e-37, 1e-30, 1e-26, 1e-23, 3e-23, 1e-22, 1e-20, 1e-19, 1e-18, 7e-16, 9e-16, 2e-15, 1e-10, 1.0, 1e10, 1e17]
    if dtype == W.WKV_F32:
        sizes += [1e-42, 1e-44]
    base = torch.randn((1, 3, 1, d), device=device, generator=g, dtype=torch.float64)
    x = torch.cat([base * f for f in sizes], 2).to(TYPES[dtype])
    x[0, 1, :, 5:] = 0.0                                       # a head of five channels
    x[0, 2, -1, : d // 2] *= 2.0 ** -8                         # and one of two sizes
    T = x.shape[2]
    keep = (x != 0).any(-1)                                    # (rows of zeros are another matter)
    pos = torch.randint(0, 5000, (1, T, axes), dtype=torch.int32, device=device, generator=g)
    axis = [i % axes for i in range(d // 2)]
    w = weights(d, dtype, device, 41)
    y, z = torch.zeros_like(x), torch.zeros_like(x)
    W.wkv_norm_rope(W.NormRopeShape(batch=1, n_tokens=T, n_q_heads=3, n_kv_heads=3, head_dim=d, dtype=dtype, inv_freq=inv, n_axes=axes, axis_of_pair=axis if axes > 1 else None,
                                    eps=eps, interleaved=interleaved), pos, w, w, x, y, x, z)
    eps32 = float(torch.tensor(eps, dtype=torch.float32))
    want, size = expected(x, w, pos, inv, axis, eps32, 1.0, interleaved)
    assert torch.isfinite(want[keep]).all()
    check(y[keep], want[keep], size[keep], dtype)
    assert torch.equal(y[keep], z[keep])
    assert int(keep.sum()) >= 3 * len(sizes) - 3
