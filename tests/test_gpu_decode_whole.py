"""wkv_decode_step_weighted with a workgroup a cache, where tests/test_decode_whole.py shows that it is chosen: more caches than the device takes at once, one full cache
among nearly empty ones, the longest caches; and the same where ranges are chosen instead."""
import pytest
import torch

import paper_2503_17922_amd as W
from tests.test_gpu_decode_weighted import Caches, check_whole

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [W.WKV_BF16, W.WKV_F16])
@pytest.mark.parametrize("B,Hq,H,d,cap", [(130, 16, 4, 128, 700), (65, 8, 8, 128, 500)])
def test_more_caches_than_run_at_once(device, dtype, B, Hq, H, d, cap):
    counts = torch.randint(0, cap, (B, H), generator=torch.Generator().manual_seed(B))
    counts[-1] = cap - 1
    c = Caches(device, counts.tolist(), Hq, H, d, dtype, cap, seed=B)
    check_whole(c)
    check_whole(c)                           # the last ones are full now


@pytest.mark.parametrize("B,Hq,H,d,cap", [(29, 16, 8, 128, 10112), (28, 8, 8, 128, 10112), (28, 8, 8, 64, 20224), (8, 32, 32, 128, 300)])
def test_one_full_cache_among_nearly_empty_ones(device, B, Hq, H, d, cap):
    counts = torch.randint(0, 9, (B, H), generator=torch.Generator().manual_seed(cap))
    counts[B // 2, H // 2] = cap - 1
    c = Caches(device, counts.tolist(), Hq, H, d, W.WKV_BF16, cap, seed=cap)
    check_whole(c)


@pytest.mark.parametrize("Hq,H,d,cap", [(8, 8, 128, 10113), (8, 8, 64, 20225), (40, 8, 128, 300)])
def test_past_the_border(device, Hq, H, d, cap):
    counts = torch.randint(0, 9, (28, H), generator=torch.Generator().manual_seed(cap))
    counts[3, 5] = cap - 1
    c = Caches(device, counts.tolist(), Hq, H, d, W.WKV_BF16, cap, seed=cap)
    c.check()
    c.check()
