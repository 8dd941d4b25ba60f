"""Calls of the 4-bit cache, eviction and sampling that are refused before a launch, and calls on a stream of their own."""
import pytest
import torch

import paper_2606_24957_amd as D

pytestmark = pytest.mark.gpu
DEV = "cuda"


def caches(B=2, n=64, H=2):
    return D.kv4_empty(B, n, H, 128, DEV)


def i32(*x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def test_refusals_of_the_4_bit_cache():
    k, v = caches()
    rows = torch.zeros(2, 4, 2, 128, dtype=torch.bfloat16, device=DEV)
    q = torch.zeros(2, 4, 8, 128, dtype=torch.bfloat16, device=DEV)
    idx, cnt = torch.zeros(2, 1, 8, dtype=torch.int32, device=DEV), torch.zeros(2, 1, dtype=torch.int32, device=DEV)
    table = torch.zeros(1, 4, dtype=torch.int32, device=DEV)
    calls = {
        "seq_lens holds 1": [lambda: D.kv4_append(rows, rows, k, v, [0]), lambda: D.kv4_append(rows, rows, k, v, i32(0)),
                             lambda: D.dense_verify_attn_kv4(q, k, v, [0]),
                             lambda: D.sparse_verify_attn_kv4(q, k, v, idx, cnt, [0])],
        "n_query holds 1": [lambda: D.kv4_append(rows, rows, k, v, [0, 0], n_query=[1]),
                            lambda: D.dense_verify_attn_kv4(q, k, v, [0, 0], n_query=i32(1))],
        "holds 1 of 2": [lambda: D.kv4_append(rows, rows, k, v, [0, 0], page_table=table),
                         lambda: D.dense_verify_attn_kv4(q, k, v, [0, 0], page_table=table),
                         lambda: D.kv_evict(k, v, idx, cnt, page_table=table),
                         lambda: D.kv4_append(rows, rows, k, D.KV4(v.data[:1], v.scales[:1]), [0, 0]),
                         lambda: D.dense_verify_attn_kv4(q, D.KV4(k.data[:1], k.scales[:1]), v, [0, 0]),
                         lambda: D.kv_evict(k, D.KV4(v.data[:1], v.scales[:1]), idx, cnt)],
        "rows must be": [lambda: D.kv4_append(rows.float(), rows, k, v, [0, 0])],
        "do not fit": [lambda: D.kv4_append(rows[..., :64], rows[..., :64], k, v, [0, 0])],
        "does not fit": [lambda: D.dense_verify_attn_kv4(q[..., :64], k, v, [0, 0])],
        "q must be": [lambda: D.dense_verify_attn_kv4(q.half(), k, v, [0, 0])],
        "out must be": [lambda: D.dense_verify_attn_kv4(q, k, v, [0, 0], out=q[:, :2])],
        "idx must be": [lambda: D.sparse_verify_attn_kv4(q, k, v, idx.long(), cnt, [0, 0])],
        "count must be": [lambda: D.sparse_verify_attn_kv4(q, k, v, idx, cnt[:1], [0, 0])],
        "device tensors": [lambda: D.kv4_append(rows, rows, k, v, torch.zeros(2, dtype=torch.int32))],
        "weights": [lambda: D.kv_evict(k, v, idx, cnt, weights=torch.zeros(2, 1, 64, device=DEV).double()),
                    lambda: D.kv_evict(k, v, idx, cnt, weights_out=torch.zeros(2, 1, 64, device=DEV))],
        "new_lens": [lambda: D.kv_evict(k, v, idx, cnt, new_lens=i32(0))],
    }
    for match, group in calls.items():
        for call in group:
            with pytest.raises(ValueError, match=match):
                call()
    with pytest.raises(D.DustinError):  # 61 + 4 positions of 64
        D.kv4_append(rows, rows, k, v, [0, 0], max_len=61)
    with pytest.raises(D.DustinError):  # more than 128 rows to a KV head
        D.dense_verify_attn_kv4(torch.zeros(2, 33, 8, 128, dtype=torch.bfloat16, device=DEV), k, v, [0, 0])


def test_refusals_of_sampling():
    logits, u = torch.zeros(2, 3, 9, device=DEV), torch.zeros(2, device=DEV)
    draft, ua = torch.zeros(2, 2, dtype=torch.int32, device=DEV), torch.zeros(2, 2, device=DEV)
    calls = {
        "logits must be": [lambda: D.sample(logits[:, 0].half(), u), lambda: D.sample(logits, u),
                           lambda: D.sample(logits[:, 0].t().contiguous().t(), u),
                           lambda: D.verify_tokens(logits[0], draft, ua, u)],
        "u must be": [lambda: D.sample(logits[:, 0], u[:1]), lambda: D.sample(logits[:, 0], u.double()),
                      lambda: D.verify_tokens(logits, draft, ua, u[:1])],
        "token must be": [lambda: D.sample(logits[:, 0], u, token=draft)],
        "probs must be": [lambda: D.sample(logits[:, 0], u, probs=logits)],
        "top_k must be": [lambda: D.sample(logits[:, 0], u, top_k=torch.zeros(2, device=DEV))],
        "temperature must be": [lambda: D.sample(logits[:, 0], u, temperature=torch.zeros(3, device=DEV))],
        "draft must be": [lambda: D.verify_tokens(logits, draft[:, :1], ua, u),
                          lambda: D.verify_tokens(logits, draft.long(), ua, u)],
        "u_accept must be": [lambda: D.verify_tokens(logits, draft, ua[:, :1], u)],
        "draft_probs must be": [lambda: D.verify_tokens(logits, draft, ua, u, draft_probs=logits)],
        "n_query holds 1": [lambda: D.verify_tokens(logits, draft, ua, u, n_query=[3])],
        "accepted must be": [lambda: D.verify_tokens(logits, draft, ua, u, accepted=u)],
    }
    for match, group in calls.items():
        for call in group:
            with pytest.raises(ValueError, match=match):
                call()
    for bad in (dict(temperature=float("nan")), dict(top_p=float("nan")), dict(min_p=float("nan"))):
        with pytest.raises(D.DustinError):
            D.sample(logits[:, 0], u, **bad)


def test_a_stream_of_their_own():
    """What a call converts (lists, strided tables and counts) and clears is in order with its launches on its stream,
    behind long work on the current one."""
    g = torch.Generator(device=DEV).manual_seed(5)
    k, v = caches(8, 16)
    rows = torch.randn(2, 40, 2, 128, generator=g, device=DEV).bfloat16()
    wide = torch.arange(16, dtype=torch.int32, device=DEV).view(2, 8)
    wide[0], wide[1] = i32(7, 0, 3, 0, 5, 0, 1, 0), i32(6, 0, 2, 0, 4, 0, 0, 0)
    table = wide[:, ::2]
    logits, u = torch.randn(2, 1003, generator=g, device=DEV), torch.rand(2, generator=g, device=DEV)
    kw = dict(n_query=[40, 33], page_table=table, max_len=0)
    D.kv4_append(rows, rows, k, v, [0, 0], **kw)
    want = D.kv4_read(k, v, [0, 0], nq_max=40, **kw) + (D.sample(logits, u, top_p=0.9),)
    torch.cuda.synchronize()
    k.data.zero_(), v.data.zero_()
    s = torch.cuda.Stream()
    busy = torch.randn(4096, 4096, device=DEV)
    torch.cuda.synchronize()
    for _ in range(4):
        busy = busy @ busy * 1e-3
    D.kv4_append(rows, rows, k, v, [0, 0], stream=s, **kw)
    got = D.kv4_read(k, v, [0, 0], nq_max=40, stream=s, **kw) + (D.sample(logits, u, top_p=0.9, stream=s),)
    s.synchronize()
    for x, y in zip(got, want):
        assert torch.equal(x.view(torch.int16) if x.dtype == torch.bfloat16 else x,
                           y.view(torch.int16) if y.dtype == torch.bfloat16 else y)
    torch.cuda.synchronize()


def test_empty_calls():
    k, v = caches()
    rows = torch.zeros(2, 0, 2, 128, dtype=torch.bfloat16, device=DEV)
    q = torch.randn(2, 3, 8, 128, device=DEV).bfloat16()
    assert D.kv4_append(rows, rows, k, v, [0, 0]) is None
    a, b = D.kv4_read(k, v, [5, 6], nq_max=0)
    assert a.shape == b.shape == (2, 0, 2, 128)
    assert D.dense_verify_attn_kv4(q[:, :0], k, v, [0, 0]).shape == (2, 0, 8, 128)
    assert D.dense_verify_attn_kv4(q[:0], k, v, []).shape == (0, 3, 8, 128)
    none = torch.zeros(2, 1, 0, dtype=torch.int32, device=DEV), torch.zeros(2, 1, dtype=torch.int32, device=DEV)
    x = torch.randn(2, 3, 2, 128, device=DEV).bfloat16()
    D.kv4_append(x, x, k, v, [0, 0])  # a selection of nothing: the window alone, at position 0
    got = D.sparse_verify_attn_kv4(q, k, v, *none, [0, 0])
    assert torch.equal(got, D.dense_verify_attn_kv4(q, k, v, [0, 0], max_len=0))
    before, lens = k.data.clone(), i32(3, 3)
    D.kv_evict(k, v, *none, new_lens=lens)
    assert torch.equal(k.data, before) and lens.tolist() == [0, 0]
    z = torch.zeros(0, device=DEV)
    assert D.sample(torch.zeros(0, 9, device=DEV), z).shape == (0,)
    acc, tok = D.verify_tokens(torch.zeros(0, 3, 9, device=DEV), torch.zeros(0, 2, dtype=torch.int32, device=DEV),
                               torch.zeros(0, 2, device=DEV), z)
    assert acc.shape == tok.shape == (0,)
    logits = torch.randn(2, 1, 9, device=DEV)
    acc, tok = D.verify_tokens(logits, torch.zeros(2, 0, dtype=torch.int32, device=DEV), torch.zeros(2, 0, device=DEV),
                               torch.zeros(2, device=DEV), temperature=0.0)
    assert acc.tolist() == [1, 1] and torch.equal(tok.long(), logits[:, 0].argmax(-1))
