"""The 4-bit cache on the GPU: append and read bit for bit against the format in float64, and the verification
attention over it (sparse and dense, contiguous and paged) against float64 attention over the cache's values."""
import numpy as np
import pytest
import torch

import paper_2606_24957_amd as D
from tests import kv4_util as U

pytestmark = pytest.mark.gpu
DEV = "cuda"


def i32(x):
    return torch.tensor(list(x), dtype=torch.int32, device=DEV)


def special_rows(shape, seed):
    """bf16 rows with blocks of every magnitude, ties, zeros, subnormals, infinities and NaN."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal(shape) * np.exp2(rng.integers(-20, 20, shape[:-1] + (1,)))
    f = x.reshape(-1, 32)
    n = f.shape[0]
    f[0 % n] = 0.0
    f[1 % n] = np.exp2(np.linspace(-133, -120, 32)) * np.where(np.arange(32) % 2, 1, -1)   # subnormals among them
    f[2 % n, :4] = [np.inf, -np.inf, np.nan, 1.0]
    f[3 % n] = np.nan
    f[4 % n] = np.tile([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.5], 4) * np.where(np.arange(32) % 3, 1, -1)  # ties
    f[5 % n] = U.BF16_MAX * np.linspace(-1, 1, 32)
    f[6 % n] = -0.0
    return torch.from_numpy(x).to(torch.bfloat16).to(DEV)


def values(cache):
    return U.decode(cache.data.cpu().numpy(), cache.scales.cpu().numpy())


def paged(rng, B, maxp, extra=3):
    return torch.from_numpy(rng.permutation(B * maxp + extra)[:B * maxp].astype(np.int32).reshape(B, maxp)).to(DEV)


def at(pt, ps, b, pos):
    pos = np.asarray(pos)
    if pt is None:
        return np.full_like(pos, b), pos
    return pt.cpu().numpy()[b][pos // ps], pos % ps


@pytest.mark.parametrize("H,d,T,ps", [(1, 128, 1, 0), (8, 128, 5, 16), (3, 64, 7, 0), (4, 128, 300, 4), (2, 64, 33, 1)])
def test_append_and_read(H, d, T, ps):
    B, cap = 3, 400
    rng = np.random.default_rng(H * d + T)
    seq, nq = [0, 17, cap - T], [T, max(1, T // 2), T]
    maxp = -(-cap // ps) if ps else 0
    pt = paged(rng, B, maxp) if ps else None
    k, v = D.kv4_empty(B, cap, H, d, DEV) if not ps else D.kv4_empty(B * maxp + 3, ps, H, d, DEV)
    for c in (k, v):  # what was there stays there
        c.data.copy_(torch.randint(0, 256, c.data.shape, dtype=torch.uint8, device=DEV))
        c.scales.copy_(torch.randint(100, 140, c.scales.shape, dtype=torch.uint8, device=DEV))
    new = special_rows((B, T, 2 * H, d), T)
    k_new, v_new = new[:, :, :H], new[:, :, H:]  # rows of a wider projection
    want = [values(k), values(v)]
    for b in range(B):
        where = at(pt, ps, b, range(seq[b], seq[b] + nq[b]))
        for w, x in zip(want, (k_new, v_new)):
            w[where] = U.rounded(x[b, :nq[b]].float().cpu().numpy())
    D.kv4_append(k_new, v_new, k, v, i32(seq), n_query=i32(nq), page_table=pt, max_len=cap - T)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(values(k), want[0])
    np.testing.assert_array_equal(values(v), want[1])
    assert int(k.scales.max()) <= 252 and int(v.scales.min()) >= 2
    outs = [torch.full((B, T, H, d), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    D.kv4_read(k, v, i32(seq), n_query=i32(nq), page_table=pt, max_len=cap - T, k_out=outs[0], v_out=outs[1])
    torch.cuda.synchronize()
    for w, o in zip(want, outs):
        for b in range(B):
            got = o[b].double().cpu().numpy()
            np.testing.assert_array_equal(got[:nq[b]], w[at(pt, ps, b, range(seq[b], seq[b] + nq[b]))])
            assert (got[nq[b]:] == 7.0).all()


def test_append_past_the_cache_writes_nothing_there():
    """Device lengths beyond the host's bound are clamped, and a position without a page is not written."""
    k, v = D.kv4_empty(4, 16, 2, 128, DEV)
    pt = i32([1]).view(1, 1)
    new = torch.ones((1, 3, 2, 128), dtype=torch.bfloat16, device=DEV)
    D.kv4_append(new, new, k, v, i32([1000]), page_table=pt, max_len=13)
    torch.cuda.synchronize()
    assert (values(k)[1, 13:] == 1).all() and values(k).sum() == 3 * 2 * 128
    D.kv4_append(new, new, k, v, i32([-5]), page_table=i32([77]).view(1, 1), max_len=13)  # a page id past the pool
    torch.cuda.synchronize()
    assert (values(v)[3, :3] == 1).all() and values(v).sum() == 2 * 3 * 2 * 128


def make(B, H, need, ps, seed, mag=1.0, tail=True):
    """Caches with rows for `need` positions per sequence; what lies behind them has scales of 2^127."""
    rng = np.random.default_rng(seed)
    cap = max(need) + 5
    maxp = -(-cap // ps) if ps else 0
    pt = paged(rng, B, maxp) if ps else None
    k, v = D.kv4_empty(B, cap, H, 128, DEV) if not ps else D.kv4_empty(B * maxp + 3, ps, H, 128, DEV)
    if tail:
        for c in (k, v):
            c.data.fill_(0x77)
            c.scales.fill_(254)
    x = torch.from_numpy(rng.standard_normal((2, B, max(need), H, 128)) * mag).to(torch.bfloat16).to(DEV)
    D.kv4_append(x[0], x[1], k, v, i32([0] * B), n_query=i32(need), page_table=pt,
                 max_len=(maxp * ps if ps else cap) - max(need))
    return k, v, pt


def check(out, q, k, v, pt, ps, seq, nq, positions, scale):
    """positions(b, g): the selected positions of a KV head, before the window."""
    Hq, H = q.shape[2], k.data.shape[2]
    gs = Hq // H
    kk, vv = values(k), values(v)
    o, qq = out.double().cpu().numpy(), q.double().cpu().numpy()
    for b in range(len(seq)):
        for g in range(H):
            sel = np.asarray(positions(b, g), dtype=np.int64)
            pos = np.concatenate((sel, np.arange(seq[b], seq[b] + nq[b])))
            if nq[b]:
                rows = tuple(at(pt, ps, b, pos)) + (np.full(len(pos), g),)
                limits = np.repeat(len(sel) + 1 + np.arange(nq[b]), gs)
                x = qq[b, :nq[b], g * gs:(g + 1) * gs].reshape(-1, 128)
                ref, tol = U.attention(x, kk[rows], vv[rows], limits, scale)
                got = o[b, :nq[b], g * gs:(g + 1) * gs].reshape(-1, 128)
                worst = (np.abs(got - ref) / tol).max()
                assert worst <= 1, f"b={b} g={g}: {worst} of the tolerance"
        assert np.isnan(o[b, nq[b]:]).all(), f"b={b}: rows past T_b were written"


DENSE = [  # Hq, Hkv, seq_lens, n_query, page size
    (8, 1, [0], [1], 0), (8, 1, [1], [1], 0), (8, 1, [127], [1], 16), (8, 8, [128, 31], [1, 1], 0),
    (28, 4, [300, 0, 129], [5, 1, 3], 16), (64, 8, [1000, 33, 2047], [9, 0, 4], 16), (16, 2, [511, 700], [6, 5], 1),
    (32, 1, [90, 257], [4, 2], 32), (48, 4, [640], [8], 0), (128, 8, [77, 3000], [8, 7], 16), (8, 1, [20000], [2], 0),
    (40, 8, [129] * 40, [1] * 40, 0), (80, 5, [63, 64, 65], [6, 6, 6], 64),
]


@pytest.mark.parametrize("Hq,H,seq,nq,ps", DENSE)
def test_dense(Hq, H, seq, nq, ps):
    B = len(seq)
    k, v, pt = make(B, H, [n + t for n, t in zip(seq, nq)], ps, sum(seq) + Hq)
    g = torch.Generator(device=DEV).manual_seed(Hq)
    q = 2 * torch.randn((B, max(nq), Hq, 128), generator=g, device=DEV, dtype=torch.bfloat16)
    out = torch.full_like(q, float("nan"))
    D.dense_verify_attn_kv4(q, k, v, i32(seq), n_query=i32(nq), page_table=pt, out=out, max_len=max(seq))
    torch.cuda.synchronize()
    check(out, q, k, v, pt, ps, seq, nq, lambda b, h: np.arange(seq[b]), 128 ** -0.5)


SPARSE = [  # Hq, Hkv, seq_lens, n_query, counts, groups, page size
    (8, 1, [2048], [5], [256], 1, 0), (28, 4, [500, 70], [4, 1], [64, 21], 1, 16), (64, 8, [900, 40], [5, 2], [333, 0], 8, 16),
    (64, 8, [4100] * 3, [9, 3, 0], [1025, 7, 90], 1, 0), (16, 16, [200], [1], [31], 16, 1), (24, 2, [99], [8], [99], 2, 0),
    (128, 8, [600, 601], [8, 8], [97, 128], 8, 32), (8, 1, [5000], [1], [4999], 1, 16),
]


@pytest.mark.parametrize("Hq,H,seq,nq,cnt,groups,ps", SPARSE)
def test_sparse(Hq, H, seq, nq, cnt, groups, ps):
    B = len(seq)
    rng = np.random.default_rng(sum(seq) + groups)
    k, v, pt = make(B, H, [n + t for n, t in zip(seq, nq)], ps, sum(seq))
    g = torch.Generator(device=DEV).manual_seed(Hq + 1)
    wide = 2 * torch.randn((B, max(nq), 2 * Hq, 128), generator=g, device=DEV, dtype=torch.bfloat16)
    q = wide[:, :, Hq:]
    idx = np.full((B, groups, max(cnt) + 3), 2 ** 30, dtype=np.int32)  # entries from count on are not positions
    counts = np.zeros((B, groups), dtype=np.int32)
    for b in range(B):
        for j in range(groups):
            c = max(0, cnt[b] - 5 * j)
            idx[b, j, :c] = np.sort(rng.choice(seq[b], c, replace=False))
            counts[b, j] = c
    ti = torch.from_numpy(idx).to(DEV)
    buf = torch.full((B, max(nq), 2 * Hq, 128), float("nan"), dtype=torch.bfloat16, device=DEV)
    out = buf[:, :, :Hq]
    D.sparse_verify_attn_kv4(q, k, v, ti, torch.from_numpy(counts).to(DEV), i32(seq), n_query=i32(nq), page_table=pt,
                             out=out, max_len=max(seq))
    torch.cuda.synchronize()
    assert torch.isnan(buf[:, :, Hq:].float()).all()
    check(out, q, k, v, pt, ps, seq, nq, lambda b, h: idx[b, h if groups > 1 else 0, :counts[b, h if groups > 1 else 0]],
          128 ** -0.5)


def test_scores_far_apart():
    """Keys whose scores rise by tens of units: the running maximum moves at many steps, and most weights vanish."""
    seq, nq = [700], [3]
    k, v, pt = make(1, 1, [703], 0, 5)
    x = torch.zeros((1, 703, 1, 128), dtype=torch.bfloat16, device=DEV)
    x[0, :, 0, :] = torch.linspace(-6, 6, 703, device=DEV)[:, None].to(torch.bfloat16)
    D.kv4_append(x, x, k, v, i32([0]), max_len=0)
    q = torch.ones((1, 3, 8, 128), dtype=torch.bfloat16, device=DEV) * torch.tensor([8.0, -8.0, 0.0], device=DEV).view(1, 3, 1, 1)
    q = q.to(torch.bfloat16)
    out = torch.full_like(q, float("nan"))
    D.dense_verify_attn_kv4(q, k, v, i32(seq), n_query=i32(nq), out=out, max_len=700)
    torch.cuda.synchronize()
    check(out, q, k, v, None, 0, seq, nq, lambda b, h: np.arange(700), 128 ** -0.5)


def test_head_major_cache_and_apart_k_and_v():
    """Other orders: [B, Hkv, N, d] storage, K and V in buffers of their own with different strides."""
    B, H, n = 2, 4, 333
    k0, v0, _ = make(B, H, [n + 2, 200], 0, 9)
    kd = k0.data.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)
    ksc = k0.scales.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)
    big = torch.zeros((B, v0.data.shape[1], H, 96), dtype=torch.uint8, device=DEV)
    big[..., 16:80] = v0.data
    k, v = D.KV4(kd, ksc), D.KV4(big[..., 16:80], v0.scales.contiguous())
    q = torch.randn((B, 2, 16, 128), device=DEV, dtype=torch.bfloat16)
    a = D.dense_verify_attn_kv4(q, k0, v0, i32([n, 198]), max_len=n)
    b = D.dense_verify_attn_kv4(q, k, v, i32([n, 198]), max_len=n)
    torch.cuda.synchronize()
    assert torch.equal(a.view(torch.int16), b.view(torch.int16))


def test_repeated_streams_and_graph():
    """The same bits again, on another stream, and from a captured graph with eager calls of another shape between."""
    seq, nq = [3000, 1500], [5, 4]
    k, v, pt = make(2, 8, [3005, 1504], 16, 21)
    q = torch.randn((2, 5, 64, 128), device=DEV, dtype=torch.bfloat16)
    out = torch.zeros_like(q)
    kw = dict(n_query=i32(nq), page_table=pt, max_len=3000)
    s, small = i32(seq), i32([100, 7])
    D.dense_verify_attn_kv4(q, k, v, s, out=out, **kw)
    torch.cuda.synchronize()
    ref = out.clone()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        call = D.plan_dense_verify_attn_kv4(q, k, v, s, out=out, **kw)
        out.zero_()
        call()
    torch.cuda.synchronize()
    assert torch.equal(out.view(torch.int16), ref.view(torch.int16))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        call()
    for _ in range(3):
        out.zero_()
        D.dense_verify_attn_kv4(q[:, :2], k, v, small, page_table=pt, max_len=100)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.view(torch.int16), ref.view(torch.int16))


def test_row_past_four_gib():
    """Rows that lie more than 2^32 bytes into the cache."""
    n = 34000000
    data = torch.zeros((1, n, 1, 2, 64), dtype=torch.uint8, device=DEV)
    scales = torch.zeros((1, n, 1, 2, 4), dtype=torch.uint8, device=DEV)
    k, v = D.KV4(data[..., 0, :], scales[..., 0, :]), D.KV4(data[..., 1, :], scales[..., 1, :])
    x = torch.randn((1, 300, 1, 128), device=DEV, dtype=torch.bfloat16)
    start = n - 400
    D.kv4_append(x, -x, k, v, i32([start]), max_len=n - 300)
    q = torch.randn((1, 1, 8, 128), device=DEV, dtype=torch.bfloat16)
    out = torch.full_like(q, float("nan"))
    idx = torch.arange(start, start + 299, dtype=torch.int32, device=DEV).view(1, 1, -1)
    D.sparse_verify_attn_kv4(q, k, v, idx, i32([299]).view(1, 1), i32([start + 299]), out=out, max_len=n - 1)
    torch.cuda.synchronize()
    rows = U.rounded(x[0, :, 0].double().cpu().numpy())
    ref, tol = U.attention(q[0, 0].double().cpu().numpy(), rows, -rows, [300] * 8, 128 ** -0.5)
    assert (np.abs(out[0, 0].double().cpu().numpy() - ref) <= tol).all()


@pytest.mark.parametrize("T,gs,paged", [(2, 4, False), (4, 8, True), (5, 8, False)])
def test_batches_that_fill_the_chip_twice(T, gs, paged):
    """Enough tokens (over 4096 granules of 128) for two workgroups on every CU, one, two and three tiles of query rows;
    a sequence that ends inside a granule and one of a single token between long ones."""
    H, lens, page = 8, [40000, 1, 27011], 64
    cap = 40000 + 64
    g = torch.Generator(device="cuda").manual_seed(T)
    per = cap // page + 1
    k, v = D.kv4_empty(3 * per if paged else 3, page if paged else cap, H, 128, "cuda")
    table = torch.randperm(3 * per, generator=g, device="cuda").int().view(3, per) if paged else None
    x = torch.randn(3, 5008, H, 128, generator=g, device="cuda").bfloat16()
    y = torch.randn(3, 5008, H, 128, generator=g, device="cuda").bfloat16()
    kw = dict(page_table=table)
    for i in range(8):
        D.kv4_append(x.roll(17 * i, 1), y.roll(5 * i, 1), k, v, [5008 * i] * 3, max_len=5008 * 7, **kw)
    q = torch.randn(3, T, H * gs, 128, generator=g, device="cuda").bfloat16()
    out = D.dense_verify_attn_kv4(q, k, v, lens, max_len=40000, **kw)
    kk, vv = D.kv4_read(k, v, [0] * 3, n_query=[n + T for n in lens], nq_max=40000 + T, max_len=0, **kw)
    torch.cuda.synchronize()
    for b, n in enumerate(lens):
        for h in (0, 3, 7):
            rows = q[b, :, h * gs:(h + 1) * gs].double().cpu().numpy().reshape(-1, 128)
            ref, tol = U.attention(rows, kk[b, :n + T, h].double().cpu().numpy(), vv[b, :n + T, h].double().cpu().numpy(),
                                   np.repeat(n + 1 + np.arange(T), gs), 128 ** -0.5)
            got = out[b, :, h * gs:(h + 1) * gs].double().cpu().numpy().reshape(-1, 128)
            assert (np.abs(got - ref) <= tol).all(), f"sequence {b} head {h}"
