"""Caches in 8 and 4 bits by their definition, on the host in 64 bits: every number of a format from a list, the scale by trying
powers of two.  Test infrastructure."""
import numpy as np
import torch

GROUP, LEAST = 32, -100
E4M3 = np.array([m * 2.0 ** -9 for m in range(8)] + [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8)][:-1])
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
TABLES = [E4M3, E2M1]            # by wkv_cache_format; a number's place is its code without the sign


def encode(rows, fmt):
    """rows [n, d] (any type) -> codes uint8 [n, bytes], scales uint8 [n, d / 32]."""
    x = np.asarray(rows.detach().double().cpu().numpy())
    table = TABLES[fmt]
    n, d = x.shape
    parts = x.reshape(n, d // GROUP, GROUP)
    with np.errstate(invalid="ignore"):
        most = np.max(np.abs(parts), -1)
        bad = ~(most <= 2.0 ** 127)
    exponent = np.full(most.shape, LEAST)
    for e in range(LEAST, 128):
        with np.errstate(invalid="ignore"):
            exponent[most > table[-1] * 2.0 ** e] = e + 1
    exponent[bad] = 0
    y = np.where(bad[..., None], 0.0, parts) / np.exp2(exponent.astype(np.float64))[..., None]
    mag = np.abs(y)
    above = np.minimum(np.searchsorted(table, mag), len(table) - 1)
    below = np.maximum(above - 1, 0)
    lo, hi = mag - table[below], table[above] - mag
    code = np.where(lo < hi, below, np.where(lo > hi, above, np.where(below % 2 == 0, below, above)))
    sign = np.signbit(y) & ~bad[..., None]
    scales = np.where(bad, 255, exponent + 127).astype(np.uint8)
    code = code.reshape(n, d)
    sign = sign.reshape(n, d)
    if fmt == 0:
        codes = (code + 128 * sign).astype(np.uint8)
    else:
        code = code + 8 * sign
        codes = (code[:, 0::2] + 16 * code[:, 1::2]).astype(np.uint8)
    return codes, scales


def decode(codes, scales, fmt):
    """What codes [n, bytes] and scales [n, d / 32] stand for, float64 [n, d]."""
    codes, scales = np.asarray(codes).astype(np.int64), np.asarray(scales).astype(np.int64)
    if fmt == 0:
        value = np.where(codes >= 128, -1.0, 1.0) * np.append(E4M3, np.nan)[codes & 127]
    else:
        half = np.stack([codes & 15, codes >> 4], -1).reshape(len(codes), -1)
        value = np.where(half >= 8, -1.0, 1.0) * E2M1[half & 7]
    scale = np.where(scales == 255, np.nan, np.exp2(scales - 127.0))
    return value * np.repeat(scale, GROUP, -1)


def decode_torch(codes, scales, fmt):
    """The same for tensors of any leading shape, on their device."""
    flat_c, flat_s = codes.reshape(-1, codes.shape[-1]).cpu().numpy(), scales.reshape(-1, scales.shape[-1]).cpu().numpy()
    v = torch.from_numpy(decode(flat_c, flat_s, fmt))
    return v.reshape(*codes.shape[:-1], -1).to(codes.device)
