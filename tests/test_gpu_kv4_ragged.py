"""4-bit caches that hold exactly what each sequence needs, where the longest sequence has the shortest window: append,
read-back and attention, contiguous and paged, with and without a stated max_len."""
import numpy as np
import pytest
import torch

import paper_2606_24957_amd as D
from tests import kv4_util as U
from tests.test_gpu_kv4 import at, check, i32, values

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("ps", [0, 16])
@pytest.mark.parametrize("stated", [False, True])
@pytest.mark.parametrize("seq,nq", [([64, 10, 37], [1, 9, 4]), ([300, 0, 291], [0, 9, 1]), ([1, 2], [2, 1])])
def test_no_room_but_each_ones_own(seq, nq, stated, ps):
    B, H, T = len(seq), 2, max(nq)
    need = [n + t for n, t in zip(seq, nq)]
    rng = np.random.default_rng(sum(need) + ps)
    if ps:
        per = [-(-n // ps) for n in need]
        perm = rng.permutation(sum(per)).astype(np.int32)
        table, first = np.zeros((B, max(per)), dtype=np.int32), 0
        for b, p in enumerate(per):
            table[b, :p] = perm[first:first + p]
            first += p
        pt = torch.from_numpy(table).to(DEV)
        k, v = D.kv4_empty(sum(per), ps, H, 128, DEV)
    else:
        pt = None
        k, v = D.kv4_empty(B, max(need), H, 128, DEV)
    x = torch.from_numpy(rng.standard_normal((2, B, max(need), H, 128))).to(torch.bfloat16).to(DEV)
    D.kv4_append(x[0], x[1], k, v, [0] * B, n_query=i32(seq), page_table=pt)  # the contexts, of lengths of their own
    win = torch.from_numpy(rng.standard_normal((2, B, T, H, 128))).to(torch.bfloat16).to(DEV)
    kw = dict(n_query=i32(nq), page_table=pt, **(dict(max_len=max(seq)) if stated else {}))
    D.kv4_append(win[0], win[1], k, v, i32(seq), **kw)
    back = D.kv4_read(k, v, i32(seq), nq_max=T, **kw)
    q = torch.randn((B, T, 4 * H, 128), device=DEV, dtype=torch.bfloat16)
    dense, sparse = torch.full_like(q, float("nan")), torch.full_like(q, float("nan"))
    D.dense_verify_attn_kv4(q, k, v, i32(seq), out=dense, **kw)
    sel = [np.arange(n)[::2] for n in seq]
    idx = np.zeros((B, 1, max(1, max(len(s) for s in sel))), dtype=np.int32)
    for b, s in enumerate(sel):
        idx[b, 0, :len(s)] = s
    D.sparse_verify_attn_kv4(q, k, v, torch.from_numpy(idx).to(DEV), i32([len(s) for s in sel]).view(B, 1), i32(seq),
                             out=sparse, **kw)
    torch.cuda.synchronize()
    for c, rows, new, got in zip((k, v), x, win, back):
        held = values(c)
        for b in range(B):
            where = at(pt, ps, b, np.arange(need[b]))
            want = np.concatenate((rows[b, :seq[b]].double().cpu().numpy(), new[b, :nq[b]].double().cpu().numpy()))
            np.testing.assert_array_equal(held[where], U.rounded(want))
            np.testing.assert_array_equal(got[b, :nq[b]].double().cpu().numpy(), held[where][seq[b]:])
    check(dense, q, k, v, pt, ps, seq, nq, lambda b, h: np.arange(seq[b]), 128 ** -0.5)
    check(sparse, q, k, v, pt, ps, seq, nq, lambda b, h: sel[b], 128 ** -0.5)


@pytest.mark.parametrize("long_k", [False, True])
def test_positions_outside_the_shorter_cache(long_k):
    """K and V of different lengths: a selected position past the shorter one counts as its last."""
    n, more, H = 60, 4000, 2
    x = torch.randn((2, 1, n + 1, H, 128), device=DEV, dtype=torch.bfloat16)
    k, v = (D.kv4_empty(1, n + 1 + (more if long_k == (i == 0) else 0), H, 128, DEV)[i] for i in range(2))
    k, v = (D.KV4(c.data.clone(), c.scales.clone()) for c in (k, v))
    D.kv4_append(x[0], x[1], k, v, [0], max_len=0)
    q = torch.randn((1, 1, 4 * H, 128), device=DEV, dtype=torch.bfloat16)
    idx = i32([3, 59, 60, 61, 4000, 2 ** 31 - 1, -5]).view(1, 1, -1)
    out = torch.full_like(q, float("nan"))
    D.sparse_verify_attn_kv4(q, k, v, idx, i32([7]).view(1, 1), i32([n]), out=out)
    torch.cuda.synchronize()
    check(out, q, k, v, None, 0, [n], [1], lambda b, h: [3, 59, 60, 60, 60, 60, 0], 128 ** -0.5)
