"""The attention over 4-bit caches as a weighted mean: where every value row is the same, that row comes back bit for
bit, whatever the weights are and however they are rounded (numerator and denominator are of the same numbers; the sums'
float32 rounding, some thousand additions of 2^-24 at most, is far below the half step of 2^-9 that would move a bf16)."""
import pytest
import torch

import paper_2606_24957_amd as D

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("B,Hq,H,T,n,ps", [(1, 8, 1, 1, 2, 0), (1, 8, 1, 1, 30000, 0), (300, 8, 1, 5, 300, 0),
                                           (32, 28, 4, 1, 700, 16), (32, 64, 8, 5, 333, 0), (16, 64, 8, 9, 1500, 16),
                                           (40, 128, 8, 8, 400, 0), (64, 48, 4, 8, 640, 16), (40, 96, 8, 8, 500, 0)])
@pytest.mark.parametrize("spread", [0.05, 1.0, 8.0])
def test_equal_values_come_back(B, Hq, H, T, n, ps, spread):
    g = torch.Generator(device=DEV).manual_seed(n + T)
    per = -(-(n + T) // ps) if ps else 0
    k, v = D.kv4_empty(B * per, ps, H, 128, DEV) if ps else D.kv4_empty(B, n + T, H, 128, DEV)
    pt = torch.randperm(B * per, generator=g, device=DEV).int().view(B, per) if ps else None
    x = torch.randn((B, n + T, H, 128), generator=g, device=DEV).bfloat16()
    y = torch.randn((B, 1, H, 128), generator=g, device=DEV).bfloat16().expand(B, n + T, H, 128).contiguous()
    D.kv4_append(x, y, k, v, [0] * B, page_table=pt, max_len=0)
    row = D.kv4_read(k, v, [0] * B, nq_max=1, page_table=pt, max_len=0)[1]  # [B, 1, H, 128]
    q = (spread * torch.randn((B, T, Hq, 128), generator=g, device=DEV)).bfloat16()
    idx = torch.arange(0, n, 2, dtype=torch.int32, device=DEV).view(1, 1, -1).expand(B, 1, (n + 1) // 2).contiguous()
    cnt = torch.full((B, 1), idx.shape[2], dtype=torch.int32, device=DEV)
    dense = D.dense_verify_attn_kv4(q, k, v, [n] * B, page_table=pt, max_len=n)
    sparse = D.sparse_verify_attn_kv4(q, k, v, idx, cnt, [n] * B, page_table=pt, max_len=n)
    torch.cuda.synchronize()
    want = row.repeat_interleave(Hq // H, 2).expand(B, T, Hq, 128)
    for out in (dense, sparse):
        wrong = int((out != want).sum())
        assert wrong == 0, f"{wrong} of {out.numel()}"
