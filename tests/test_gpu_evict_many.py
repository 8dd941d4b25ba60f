"""Eviction of more rows than one launch's grid counts: long selections of many sequences, few of them kept."""
import pytest
import torch

import paper_2606_24957_amd as D

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("B", [80, 130, 300])
def test_many_long_selections(B, four):
    H, ps, k_max, pool = 8, 16, 131072, 64
    g = torch.Generator(device=DEV).manual_seed(B)
    make = (lambda n: D.kv4_empty(n, ps, H, 128, DEV)) if four else (
        lambda n: tuple(torch.zeros((n, ps, H, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2)))
    parts = lambda c: list(c) if four else [c.view(torch.int16)]
    k, v = make(pool)
    for c in (k, v):
        for x in parts(c):
            x.copy_(torch.randint(0, 200, x.shape, generator=g, device=DEV).to(x.dtype))
    ko, vo = make(B)
    src = torch.randint(0, pool, (B, k_max // ps), generator=g, device=DEV).int()
    dst = torch.arange(B, dtype=torch.int32, device=DEV).view(B, 1).expand(B, k_max // ps).contiguous()
    cnt = torch.randint(0, ps + 1, (B, 1), generator=g, device=DEV).int()
    idx = torch.zeros((B, 1, k_max), dtype=torch.int32, device=DEV)
    idx[:, 0, :ps] = torch.sort(torch.randint(0, k_max, (B, ps), generator=g, device=DEV)).values.int()
    lens = torch.full((B,), -1, dtype=torch.int32, device=DEV)
    D.kv_evict(k, v, idx, cnt, k_out=ko, v_out=vo, page_table=src, out_page_table=dst, new_lens=lens)
    torch.cuda.synchronize()
    assert torch.equal(lens, cnt[:, 0])
    at = idx[:, 0, :ps].long()
    kept = (torch.arange(ps, device=DEV) < cnt).view(B, ps, 1, 1)
    for a, b in ((k, ko), (v, vo)):
        for x, y in zip(parts(a), parts(b)):
            rows = x[src.long().gather(1, at // ps), at % ps]  # [B, ps, H, bytes]
            assert torch.equal(y, torch.where(kept, rows, torch.zeros_like(rows)))
