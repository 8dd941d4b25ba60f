"""Eviction: kept rows of bf16 and 4-bit caches to others and in place, with the weights and lengths, bit for bit."""
import numpy as np
import pytest
import torch

import paper_2606_24957_amd as D

pytestmark = pytest.mark.gpu
DEV = "cuda"


def i32(x):
    return torch.tensor(list(x), dtype=torch.int32, device=DEV)


def make(kind, B, n, H, d, ps, rng):
    maxp = -(-n // ps) if ps else 0
    lead = (B * maxp + 2, ps) if ps else (B, n)
    pt = torch.from_numpy(rng.permutation(B * maxp).astype(np.int32).reshape(B, maxp)).to(DEV) if ps else None
    if kind == "bf16":
        kv = [torch.from_numpy(rng.integers(-30000, 30000, lead + (H, d)).astype(np.int16)).to(DEV).view(torch.bfloat16)
              for _ in range(2)]
    else:
        kv = list(D.kv4_empty(*lead, H, d, DEV))
        for c in kv:
            c.data.copy_(torch.from_numpy(rng.integers(0, 256, c.data.shape).astype(np.uint8)))
            c.scales.copy_(torch.from_numpy(rng.integers(2, 250, c.scales.shape).astype(np.uint8)))
    return kv, pt


def parts(c):
    return list(c) if isinstance(c, D.KV4) else [c.view(torch.int16)]


def selection(rng, seq, cnt, groups):
    kmax = max(max(cnt), 1) + 2
    idx = np.full((len(seq), groups, kmax), -7, dtype=np.int32)
    for b, (n, c) in enumerate(zip(seq, cnt)):
        for j in range(groups):
            idx[b, j, :c] = np.sort(rng.choice(n, c, replace=False))
    return torch.from_numpy(idx).to(DEV), torch.tensor([[c] * groups for c in cnt], dtype=torch.int32, device=DEV)


def expect(src, dst, pt, opt, ps, idx, cnt, H):
    """dst after the move, from host copies."""
    s, d = src.cpu().numpy(), dst.cpu().numpy().copy()
    I, C = idx.cpu().numpy(), cnt.cpu().numpy()

    def at(table, b, pos):
        if table is None:
            return np.full_like(pos, b), pos
        return table.cpu().numpy()[b][pos // ps], pos % ps

    for b in range(I.shape[0]):
        for h in range(H):
            j = h if I.shape[1] > 1 else 0
            pos, to = I[b, j, :C[b, j]].astype(np.int64), np.arange(C[b, j])
            d[at(opt, b, to) + (np.full_like(to, h),)] = s[at(pt, b, pos) + (np.full_like(pos, h),)]
    return d


CASES = [  # kind, Hkv, d, seq_lens, counts, groups, page size
    ("bf16", 8, 128, [100, 37], [50, 37], 1, 0), ("bf16", 1, 64, [1], [1], 1, 0), ("bf16", 4, 128, [9000], [5000], 1, 16),
    ("bf16", 4, 64, [300, 0, 257], [128, 0, 256], 4, 16), ("kv4", 8, 128, [4000, 100], [2100, 21], 1, 0),
    ("kv4", 4, 128, [700, 64], [65, 64], 4, 16), ("kv4", 2, 64, [513], [512], 1, 4), ("kv4", 1, 128, [20000], [17000], 1, 0),
]


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("kind,H,d,seq,cnt,groups,ps", CASES)
def test_evict(kind, H, d, seq, cnt, groups, ps, in_place):
    rng = np.random.default_rng(sum(seq) + d)
    B, n = len(seq), max(seq)
    (k, v), pt = make(kind, B, n, H, d, ps, rng)
    idx, count = selection(rng, seq, cnt, groups)
    if in_place:  # no more rows than the cache has
        idx = idx[:, :, :min(idx.shape[2], n)]
    kmax = idx.shape[2]
    w = torch.rand((B, groups, n + 1), device=DEV)
    lens = i32([-1] * B)
    if in_place:
        ko, vo, opt, wo = k, v, pt, w
    else:
        (ko, vo), opt = make(kind, B, kmax, H, d, ps, rng)
        wo = torch.full((B, groups, kmax), -1.0, device=DEV)
    want = [expect(s, o, pt, opt, ps, idx, count, H) for a, b in ((k, ko), (v, vo)) for s, o in zip(parts(a), parts(b))]
    wwant = wo.cpu().numpy().copy()
    for b in range(B):
        for j in range(groups):
            wwant[b, j, :cnt[b]] = w.cpu().numpy()[b, j][idx.cpu().numpy()[b, j, :cnt[b]]]
    kw = {} if in_place else dict(k_out=ko, v_out=vo, out_page_table=opt, weights_out=wo)
    D.kv_evict(k, v, idx, count, page_table=pt, weights=w, new_lens=lens, **kw)
    torch.cuda.synchronize()
    for got, ref in zip([x for c in (ko, vo) for x in parts(c)], want):
        np.testing.assert_array_equal(got.cpu().numpy(), ref)
    np.testing.assert_array_equal(wo.cpu().numpy(), wwant)
    assert lens.tolist() == cnt


def test_lengths_alone_and_counts_out_of_range():
    """No kept row; a count past k_max, positions outside the cache: clamped, in bounds."""
    rng = np.random.default_rng(3)
    (k, v), _ = make("bf16", 2, 64, 2, 128, 0, rng)
    (ko, vo), _ = make("bf16", 2, 8, 2, 128, 0, rng)
    idx = i32([0, 3, 1 << 30, -4, 60, 61, 62, 63] * 2).view(2, 1, 8)
    lens = i32([5, 5])
    D.kv_evict(k, v, idx, i32([1 << 20, -3]).view(2, 1), k_out=ko, v_out=vo, new_lens=lens)
    torch.cuda.synchronize()
    assert lens.tolist() == [8, 0]
    rows = [0, 3, 63, 0, 60, 61, 62, 63]
    assert torch.equal(ko[0].view(torch.int16), k[0, rows].view(torch.int16))


def test_scores_choose_what_stays():
    """Accumulated attention weight -> selection -> eviction -> attention over the shorter cache equals the sparse
    attention over the longer one's selection, bit for bit."""
    from paper_2606_24957_amd import workloads as W
    s = W.config("qwen7b").replace(layers=1, seq_lens=(3000, 1200, 900, 64), budget=(512,) * 4, m=(0,) * 4)
    L = W.make_layer(s, 0, DEV)
    seq = i32(s.seq_lens)
    w = D.score(L.q[:, :4].contiguous(), L.k, seq, list(range(28)), max_len=3000)
    idx, cnt = D.topk(None, w, seq, 512)
    ref = D.sparse_verify_attn(L.q, L.k, L.v, idx, cnt, seq, max_len=3000)
    win = [torch.stack([c[b, n:n + 5] for b, n in enumerate(s.seq_lens)]) for c in (L.k, L.v)]
    D.kv_evict(L.k, L.v, idx, cnt, weights=w, new_lens=seq)
    D.kv_append(win[0], win[1], L.k, L.v, seq, max_len=512)
    every = torch.arange(512, dtype=torch.int32, device=DEV).view(1, 1, -1).expand(4, 1, 512).contiguous()
    out = D.sparse_verify_attn(L.q, L.k, L.v, every, cnt, seq, max_len=3000)
    torch.cuda.synchronize()
    assert seq.tolist() == [512, 512, 512, 64]
    assert torch.equal(out.view(torch.int16), ref.view(torch.int16))
