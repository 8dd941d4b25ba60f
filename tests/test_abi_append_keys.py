"""The append of keys alone: host validation of the built library (no GPU)."""
import ctypes
import os

import pytest
import torch

import paper_2606_24957_amd as D

FAKE = 0x10000  # a non-null, 256-byte aligned address that validation never dereferences


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(D.LIB_PATH):
        pytest.skip("libdustin.so not built")
    return D.lib()


def test_v_may_be_absent(L):
    kv, bt, r = D.DustinKV(), D.DustinBatch(), ctypes.byref
    kv.data, kv.num_kv_heads, kv.head_dim, kv.capacity = FAKE, 2, 128, 200
    kv.stride_h, kv.stride_n, kv.stride_b = 128, 256, 200 * 256
    bt.batch, bt.max_len, bt.nq_max, bt.seq_lens = 0, 100, 4, FAKE
    rows = (FAKE, 1024, 256, 128)
    none = (None, 0, 0, 0)
    assert L.dustin_kv_append(*rows, *none, r(kv), None, r(bt), None) == D.OK  # (an empty batch: nothing is launched)
    assert L.dustin_kv_append(*rows, *rows, r(kv), r(kv), r(bt), None) == D.OK
    bt.batch = 2
    assert L.dustin_kv_append(*rows, *rows, r(kv), None, r(bt), None) == D.ERR_INVALID_ARG
    assert L.dustin_kv_append(*rows, *none, r(kv), r(kv), r(bt), None) == D.ERR_INVALID_ARG
    assert L.dustin_kv_append(*none, *none, None, None, r(bt), None) == D.ERR_INVALID_ARG
    bt.max_len = 197
    assert L.dustin_kv_append(*rows, *none, r(kv), None, r(bt), None) == D.ERR_INVALID_ARG  # 201 positions of 200


@pytest.mark.gpu
@pytest.mark.parametrize("ps", [0, 16])
@pytest.mark.parametrize("H,d,T", [(1, 64, 1), (8, 128, 5), (40, 128, 16)])
def test_keys_alone(H, d, T, ps):
    B, cap = 3, 64
    g = torch.Generator(device="cuda").manual_seed(H + T)
    k = torch.randn((B * cap // ps, ps, H, d) if ps else (B, cap, H, d), generator=g, device="cuda").bfloat16()
    pt = torch.randperm(B * cap // ps, generator=g, device="cuda").int().view(B, -1) if ps else None
    rows = torch.randn((B, T, H, d), generator=g, device="cuda").bfloat16()
    seq, nq = torch.tensor([0, 11, cap - T]).int().cuda(), torch.tensor([T, T // 2, T]).int().cuda()
    want = k.clone()
    other = torch.zeros_like(k)
    D.kv_append(rows, rows, want, other, seq, n_query=nq, page_table=pt)
    D.kv_append(rows, None, k, None, seq, n_query=nq, page_table=pt)
    torch.cuda.synchronize()
    assert torch.equal(k.view(torch.int16), want.view(torch.int16))
    with pytest.raises(ValueError, match="v_new goes with v"):
        D.kv_append(rows, None, k, other, seq)


@pytest.mark.gpu
def test_the_step_names_no_cache_twice(monkeypatch):
    """Every append that a step over 4-bit layers plans writes its caches once."""
    from paper_2606_24957_amd import step as S
    from paper_2606_24957_amd import workloads as W

    s = W.config("tiny")
    layer = W.make_layer(s, 0, "cuda")
    est = W.make_estimation(s, layer, "cuda")
    caches = []
    for name in ("plan_kv_append", "plan_kv4_append"):
        plan = getattr(S, name)
        monkeypatch.setattr(S, name, lambda kn, vn, k, v, *a, plan=plan, **kw: (caches.append((k, v)), plan(kn, vn, k, v, *a, **kw))[1])
    S.VerifyStep(s, [S.layer4(s, layer)], est, "cuda", windows=[S.window_kv(s, layer)], score_k=layer.k)
    assert len(caches) == 2 and all(k is not v for k, v in caches)
