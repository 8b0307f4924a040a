"""The host's definition of rows in 8 and 4 bits against torch's 8-bit type, by hand, and by its bounds (no GPU)."""
import numpy as np
import pytest
import torch

from tests import few_bits as F


def test_e4m3_codes_are_torchs():
    codes = torch.arange(256, dtype=torch.uint8)
    want = codes.view(torch.float8_e4m3fn).double().numpy()
    got = F.decode(codes.numpy()[:, None].repeat(32, 1), np.full((256, 1), 127), 0)[:, 0]
    assert np.array_equal(got, want, equal_nan=True)


def test_by_hand():
    # largest 6: a scale of 1; ties go to the even code (2.5 -> 2, 3.5 -> 4, 5 -> 4, 0.25 -> 0, 0.75 -> 1, 1.25 -> 1, 1.75 -> 2)
    row = torch.tensor([[6.0, -6.0, 2.5, -3.5, 5.0, 0.25, 0.75, 1.25, 1.75, -0.25, 0.5, 1.5, 3.0, 4.0] + [0.0] * 18])
    codes, scales = F.encode(row, 1)
    assert scales.tolist() == [[127]]
    assert F.decode(codes, scales, 1)[0, :14].tolist() == [6.0, -6.0, 2.0, -4.0, 4.0, 0.0, 1.0, 1.0, 2.0, 0.0, 0.5, 1.5, 3.0, 4.0]
    assert codes[0, 0] == 7 + 16 * 15
    # anything above 6 takes the next power of two
    assert F.encode(torch.full((1, 32), 6.0 + 2 ** -20), 1)[1].tolist() == [[128]]
    assert F.encode(torch.full((1, 32), 448.0), 0)[1].tolist() == [[127]] and F.encode(torch.full((1, 32), 449.0), 0)[1].tolist() == [[128]]
    assert F.encode(torch.zeros((1, 32)), 0)[1].tolist() == [[27]]
    for x in (float("inf"), float("nan"), 2.0 ** 127 * 1.01):
        row = torch.ones((1, 64)); row[0, 5] = x
        codes, scales = F.encode(row, 0)
        assert scales[0].tolist() == [255, 119] and not codes[0, :32].any()
    assert F.encode(torch.full((1, 32), 2.0 ** 127), 0)[1].tolist() == [[246]]


@pytest.mark.parametrize("fmt,bits", [(0, 3), (1, 1)])
def test_a_value_is_off_by_half_a_step(fmt, bits):
    x = torch.randn((200, 128), generator=torch.Generator().manual_seed(1)) * torch.exp(3 * torch.randn((200, 1), generator=torch.Generator().manual_seed(2)))
    codes, scales = F.encode(x, fmt)
    v = F.decode(codes, scales, fmt)
    x = x.double().numpy()
    scale = np.repeat(np.exp2(scales.astype(np.int64) - 127.0), 32, -1)
    least = 2.0 ** -6 if fmt == 0 else 1.0
    step = np.exp2(np.floor(np.log2(np.maximum(np.abs(x) / scale, least)))) * 2.0 ** -bits * scale
    assert (np.abs(v - x) <= step / 2 * (1 + 1e-12)).all()
    most = np.abs(x).reshape(200, 4, 32).max(-1)
    top = F.TABLES[fmt][-1] * np.exp2(scales.astype(np.int64) - 127.0)
    assert (most <= top).all() and (most > top / 2).all()
