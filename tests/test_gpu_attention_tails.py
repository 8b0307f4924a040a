"""wkv_prefill_attention where one key outweighs all others and its value is zero, so that the output is what the small probabilities make of it.

A probability of a 16-bit type is rounded by half a step of its own, in fp16 by no less than 2^-25 of the units it is held in: these make the largest probability
of a row 2^13 or more, so at most 2^-38 of a row's sum is lost a key, and m keys lose m 2^-38 |v|.  The rounding of an output in fp16 has room for that: the
tolerance of `check` holds 2^-24 for it, of which subnormal results use 2^-25, and 4097 keys of mean magnitude below 1 lose less than 2^-26."""
import pytest
import torch

import paper_2503_17922_amd as W
from tests.test_gpu_prefill_attention import TYPES, run

pytestmark = pytest.mark.gpu


def one_key_on_top(gap, at, d):
    """Logits of key `at` lie `gap` (base e) above those of the others, which have a standard deviation of about a half."""
    def change(qs, ks, vs):
        for q, k, v in zip(qs, ks, vs):
            q.mul_(0.5)
            q[:, :, 0], k[:, :, 0] = 8.0, 0.0
            k[:, at, :], v[:, at, :] = 0.0, 0.0
            k[:, at, 0] = gap * d ** 0.5 / 8.0
    return change


# (query heads, KV heads, query rows, keys): blocks of 256 rows and of 128, whole and shared by several workgroups
CUTS = [(32, 8, 400, 400), (8, 2, 1100, 1100), (4, 1, 3, 4097), (32, 8, 250, 4000), (8, 8, 4097, 4097)]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("gap", [10.0, 14.0, 17.0, 20.0])
def test_a_key_of_no_value_outweighs_the_others(device, dtype, d, gap):
    for Hq, H, n, m in CUTS:
        batch = 8 if (n, m) == (400, 400) else 1
        run(device, [n] * batch, [m] * batch, Hq, H, d, dtype, lse_rows=5, seed=int(gap) + m, change=one_key_on_top(gap, 0, d))


@pytest.mark.parametrize("dtype", [W.WKV_F16, W.WKV_BF16])
@pytest.mark.parametrize("at", [1, 63, 64, 700, 1299])
def test_wherever_it_stands(device, dtype, at):
    run(device, [1300], [1300], 8, 2, 128, dtype, lse_rows=5, seed=at, change=one_key_on_top(16.0, at, 128))
    run(device, [2], [1300], 8, 2, 64, dtype, lse_rows=2, seed=at, change=one_key_on_top(18.0, at, 64))


@pytest.mark.parametrize("dtype", [W.WKV_F16, W.WKV_BF16])
def test_logits_that_rise_slowly(device, dtype):
    """Every row's largest logit lies up to some thousand steps of the reference's moves above its first."""
    def change(qs, ks, vs):
        for q, k, v in zip(qs, ks, vs):
            q.mul_(0.25)
            q[:, :, 0] = 16.0
            k[:, :, 0] = torch.linspace(-40.0, 40.0, k.shape[1], device=k.device)
            v[:, -200:] = 0.0                # (the last rows' output is the tail of their probabilities)
    for Hq, H, n, m in CUTS[1:]:
        run(device, [n], [m], Hq, H, 128, dtype, lse_rows=5, change=change)
