"""wkv_decode_step_quantized and wkv_decode_tree over caches past the memory-side cache (256 MiB), with heads, sequences and rows more than 2^32 bytes apart; and rows back
from 64 channels and for several pairs of sequence and KV head at once."""
import pytest
import torch

import paper_2503_17922_amd as W
from tests import few_bits as F
from tests.test_gpu_decode_quantized import FORMATS, TYPES, Step
from tests.test_gpu_quantized_rows import caches
from tests.test_gpu_tree import Tree, some_tree

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("d,cap", [(64, 600000), (128, 300000)])
@pytest.mark.parametrize("G", [3, 8])
def test_caches_past_the_memory_side_cache(device, fmt, dtype, d, cap, G):
    cap *= 2 if fmt == W.WKV_CACHE_E2M1 else 1
    row = (d if fmt == W.WKV_CACHE_E4M3 else d // 2) + d // 32
    assert 2 * 4 * cap * row > 256 << 20
    s = Large(device, [[4128, 0], [777, 9001]], 2 * G, 2, d, dtype, fmt, cap, seed=G)
    s.check()


class Large(Step):
    """Caches whose rows behind the counts are left out of comparisons and of the making: they are empty."""

    def __init__(self, device, counts, Hq, H, d, dtype, fmt, cap, seed, strides=None):
        most = max(max(n) for n in counts) + 1
        super().__init__(device, counts, Hq, H, d, dtype, fmt, most, seed=seed)
        B, row = len(counts), self.kc.shape[-1]
        sb, sh, st = strides or (H * cap * row, cap * row, row)
        for name in ("kc", "vc"):
            small = getattr(self, name)
            view = torch.empty((B - 1) * sb + (H - 1) * sh + (cap - 1) * st + row, dtype=torch.uint8, device=device).as_strided((B, H, most, row), (sb, sh, st, 1))
            view.copy_(small)
            setattr(self, name, view)
        for name in ("ks", "vs"):
            small = getattr(self, name)
            view = torch.empty((B, H, cap, d // 32), dtype=torch.uint8, device=device)[:, :, :most]
            view.copy_(small)
            setattr(self, name, view)
        self.shape = W.QuantizedShape(batch=B, n_q_heads=Hq, n_kv_heads=H, head_dim=d, dtype=dtype, format=fmt, capacity=cap, code_strides=(sb, sh, st))
        self.ws = torch.full((W.wkv_decode_quantized_workspace_bytes(self.shape),), 0xff, dtype=torch.uint8, device=device)


FAR = (1 << 32) + (1 << 20)


@pytest.mark.parametrize("fmt,dtype,d,cap,strides", [
    (W.WKV_CACHE_E4M3, W.WKV_BF16, 128, 500, (2 * FAR, FAR, 128)),                       # heads and sequences
    (W.WKV_CACHE_E2M1, W.WKV_F16, 64, 500, (2 * FAR, FAR, 48)),
    (W.WKV_CACHE_E4M3, W.WKV_F32, 128, 300, (128, 256, (1 << 26) - 16)),                 # rows: 300 of them, 20 GB
    (W.WKV_CACHE_E2M1, W.WKV_BF16, 128, 300, (64, 128, (1 << 26) - 16))])
def test_codes_past_32_bits(device, fmt, dtype, d, cap, strides):
    s = Large(device, [[299, 100], [40, 298]], 8, 2, d, dtype, fmt, cap, seed=70, strides=strides)
    reach = strides[0] + strides[1] if strides[0] > 1 << 32 else 298 * strides[2]
    assert reach > 1 << 32
    s.check()
    del s
    torch.cuda.empty_cache()


def far_view(x, strides, device):
    """x at strides of elements, whatever is between uninitialised."""
    size = sum((n - 1) * st for n, st in zip(x.shape, strides)) + 1
    view = torch.empty(size, dtype=x.dtype, device=device).as_strided(x.shape, strides)
    view.copy_(x)
    return view


@pytest.mark.parametrize("dtype,d,cap,c_st,n_st,counts", [
    (W.WKV_BF16, 128, 400, (1 << 32, (1 << 31) + 4096, 136), ((1 << 31) + 4096, 64 * 256, 256), [300, 130]),       # sequences and heads of caches and of new rows
    (W.WKV_F32, 64, 400, (1 << 31, (1 << 30) + 4096, 64), ((1 << 30) + 4096, 64 * 128, 64), [300, 130]),
    (W.WKV_F16, 64, 300, (64, 128, (1 << 24) - 64), (64 * 128, 64 * 128 * 4, 64), [280, 7]),                        # rows of a cache: 296 of them, 9.9 GB
    (W.WKV_BF16, 128, 5000, (128, 256, 1 << 20), (64 * 256, 64 * 256 * 4, 256), [4900, 4097])])                     # in several ranges
def test_trees_past_32_bits(device, dtype, d, cap, c_st, n_st, counts):
    T, Hq, H = 16, 4, 2
    s = Tree(device, counts, [some_tree(T, b) for b in range(2)], Hq, H, d, dtype, cap, seed=71, layout="heads")
    size = s.q.element_size()
    assert max((c_st[0] + c_st[1]) * size, (max(counts) + T - 1) * c_st[2] * size) > 1 << 32
    s.q, s.kn, s.vn = (far_view(x, n_st + (1,), device) for x in (s.q, s.kn, s.vn))
    s.out = far_view(s.out, n_st + (1,), device)
    s.kc, s.vc = ([far_view(c, c_st + (1,), device) for c in cs] for cs in (s.kc, s.vc))
    s.shape = W.TreeShape(batch=2, n_q_heads=Hq, n_kv_heads=H, head_dim=d, dtype=dtype, n_nodes=T, capacity=cap, cache_strides=c_st, q_strides=n_st, new_strides=n_st, out_strides=n_st)
    s.ws = torch.full((W.wkv_tree_workspace_bytes(s.shape),), 0xff, dtype=torch.uint8, device=device)
    s.check()
    was = [c[0].clone() for c in (s.kc, s.vc)]
    path = torch.tensor([[1, 4, 9] + [-1] * (T - 3)] * 2, dtype=torch.int32, device=device)
    W.wkv_tree_accept(s.shape, s.kc, s.vc, path, torch.tensor([3, 2], dtype=torch.int32, device=device), s.n)
    for c, w in zip((s.kc[0], s.vc[0]), was):
        for b, n in enumerate(counts):
            for i, node in enumerate([1, 4, 9][:3 - b]):
                w[b, :, n + i] = w[b, :, n + node]
        assert torch.equal(torch.isnan(c), torch.isnan(w)) and torch.equal(c.nan_to_num(), w.nan_to_num())
    assert s.n.tolist() == [[counts[0] + 3] * H, [counts[1] + 2] * H]
    del s, was
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("n_rows", [1, 2, 5, 16, 17, 30, 32, 33, 70])
def test_rows_back(device, dtype, d, fmt, n_rows):
    B, H, cap = 7, 3, 41                                       # 21 pairs: no multiple of any number of pairs to a workgroup but of one, three and seven
    g = torch.Generator(device=device).manual_seed(80 + n_rows)
    (kc,), (ks,), strides, row = caches(B, H, cap, d, fmt, device, pad=16)
    (vc,), (vs,), _, _ = caches(B, H, cap, d, fmt, device, pad=16)
    for c, s in ((kc, ks), (vc, vs)):
        c.copy_(torch.randint(0, 256, c.shape, device=device, generator=g))
        if fmt == W.WKV_CACHE_E4M3:
            c[(c & 127) == 127] = 0                            # (that code is no number)
        s.copy_(torch.randint(100, 160, s.shape, device=device, generator=g))
    s[2, 1, 3, 1] = 255                                        # a group that stands for NaN
    first = torch.randint(-5, cap + 3, (B, H), dtype=torch.int32, device=device, generator=g)
    valid = torch.randint(-1, cap + 9, (B, H), dtype=torch.int32, device=device, generator=g)
    shape = W.QuantizedShape(batch=B, n_kv_heads=H, head_dim=d, dtype=dtype, format=fmt, capacity=cap, code_strides=strides, n_rows=n_rows, row_strides=(n_rows * H * d, d, H * d))
    out = [torch.full((B, n_rows, H, d), 7.0, dtype=TYPES[dtype], device=device) for _ in range(2)]
    W.wkv_cache_dequantize(shape, [kc], [ks], [vc], [vs], first, valid, out[:1], out[1:])
    torch.cuda.synchronize()
    place = first[..., None] + torch.arange(n_rows, device=device)
    there = (place >= 0) & (place < valid[..., None].clamp(max=cap))
    for x, c, s in ((out[0], kc, ks), (out[1], vc, vs)):
        values = F.decode_torch(c[..., :row], s, fmt)
        if dtype == W.WKV_F16:
            values = torch.where(torch.isnan(values), values, values.clamp(-65504.0, 65504.0))
        want = torch.gather(values, 2, place.clamp(0, cap - 1).long()[..., None].expand(-1, -1, -1, d))
        want = torch.where(there[..., None], want, 7.0).transpose(1, 2)
        # exact in bf16 and fp32, one rounding in fp16: as torch rounds a number of 64 bits
        assert torch.equal(torch.isnan(x), torch.isnan(want))
        assert torch.equal(torch.nan_to_num(x), torch.nan_to_num(want.to(TYPES[dtype])))
