"""wkv_prefill_attention where some sequences of a batch have no rows and the others' keys are shared among workgroups: outputs, normalisers, and what lies
behind the workspace."""
import pytest
import torch

import paper_2503_17922_amd as W
from tests.test_gpu_prefill_attention import TYPES, check, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("q_len,k_len", [([0, 1, 0, 0], [5, 9000, 0, 70]), ([1] + [0] * 63, [9000] + [0] * 63), ([0, 200, 0, 3, 0], [0, 5000, 6000, 3, 1])])
def test_idle_sequences(device, dtype, q_len, k_len):
    run(device, q_len, k_len, 8, 2, 128, dtype, lse_rows=4)
    run(device, q_len, k_len, 3, 3, 64, dtype, layout="packed", lse_rows=4)


@pytest.mark.parametrize("dtype", list(TYPES))
def test_no_byte_behind_the_workspace(device, dtype):
    Hq, H, d, q_len, k_len = 8, 8, 64, [0, 3, 0, 130, 0], [9, 7000, 0, 130, 4]
    g = torch.Generator(device=device).manual_seed(8)
    q = torch.randn((5, Hq, 130, d), device=device, generator=g).to(TYPES[dtype])
    k, v = (torch.randn((5, H, 7000, d), device=device, generator=g).to(TYPES[dtype]) for _ in range(2))
    out, lse = torch.zeros_like(q), torch.zeros((5, Hq, 6), device=device)
    shape = W.AttentionShape(q_len=q_len, k_len=k_len, n_q_heads=Hq, n_kv_heads=H, head_dim=d, dtype=dtype, lse_rows=6)
    size = W.wkv_attention_workspace_bytes(shape)
    assert size > 256                        # (the work is cut)
    memory = torch.full((size + (64 << 20),), 0x5a, dtype=torch.uint8, device=device)
    W.wkv_prefill_attention(shape, q, k, v, out, lse, memory[:size])
    assert (memory[size:] == 0x5a).all()
    for b, (n, m) in enumerate(zip(q_len, k_len)):
        check(out[b, :, :n], lse[b], q[b, :, :n], k[b, :, :m], v[b, :, :m], d ** -0.5, dtype, f"sequence {b}")
        assert (out[b, :, n:] == 0).all() and (lse[b, :, :max(6 - n, 0)] == -float("inf")).all()
