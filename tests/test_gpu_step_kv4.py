"""A verification step over 4-bit caches, the verification of its drafts, the commit and the eviction, run together as a
serving loop runs them: against the bf16 step on the same values, and again after the eviction."""
import numpy as np
import pytest
import torch

import paper_2606_24957_amd as D
from paper_2606_24957_amd import step as S
from paper_2606_24957_amd import workloads as W
from tests import kv4_util as U
from tests import sample_util as SU

pytestmark = pytest.mark.gpu
DEV = "cuda"


def build(paged):
    s = W.config("ragged" if paged else "qwen7b")
    if paged:
        s = s.replace(B=3, seq_lens=(3000, 1200, 2100), n_query=(5, 3, 4), budget=(300, 128, 256), m=(140, 54, 118),
                      planted=(30, 12, 21), layers=2)
    else:
        s = s.replace(B=2, seq_lens=(2000, 700), n_query=(5, 5), budget=(256, 256), m=(118, 118), planted=(20,), layers=2)
    layers = [W.make_layer(s, l, DEV) for l in range(s.layers)]
    est = W.make_estimation(s, layers[0], DEV)
    return s, layers, est


def rounded_layer(s, layer, four):
    """The bf16 layer that holds the 4-bit one's values."""
    rows = [x + y for x, y in zip(s.seq_lens, s.n_query)]
    kk, vv = D.kv4_read(four.k, four.v, [0] * s.B, n_query=rows, nq_max=max(rows), page_table=four.page_table, max_len=0)
    k, v = layer.k.clone(), layer.v.clone()
    D.kv_append(kk, vv, k, v, torch.zeros(s.B, dtype=torch.int32, device=DEV),
                n_query=torch.tensor(rows, dtype=torch.int32, device=DEV), page_table=layer.page_table, max_len=0)
    return W.Layer(layer.q, k, v, layer.page_table)


@pytest.mark.parametrize("paged", [False, True])
def test_step_accept_evict_step(paged):
    s, layers, est = build(paged)
    windows = [S.window_kv(s, l) for l in layers]
    four = [S.layer4(s, l) for l in layers]
    plain = [rounded_layer(s, l, f) for l, f in zip(layers, four)]
    score_k = layers[0].k.clone()
    st4 = S.VerifyStep(s, four, est, DEV, windows=windows, score_k=score_k)
    st16 = S.VerifyStep(s, plain, est, DEV, windows=[S.window_kv(s, p) for p in plain], score_k=layers[0].k.clone())
    st4.run()
    st16.run()
    torch.cuda.synchronize()
    assert torch.equal(st4.cnt, st16.cnt)
    for b in range(s.B):
        c = int(st4.cnt[b, 0])
        assert torch.equal(st4.idx[b, 0, :c], st16.idx[b, 0, :c])
    # the same sums over the same values, each within the attention's rounding (two roundings of the probabilities, two
    # of the output: 4 * 2^-8 of the magnitudes)
    for l, (a, c) in enumerate(zip(st4.outs, st16.outs)):
        for b, t in enumerate(s.n_query):
            x, y = a[b, :t].float(), c[b, :t].float()
            v = plain[l].contiguous_kv(s)[1][b, :s.seq_lens[b] + t].float().abs().amax()
            assert (x - y).abs().max() <= 4 * 2.0 ** -8 * 2 * v, f"layer {l} sequence {b}"

    # the drafts against the target's logits, and the accepted tokens kept
    g = torch.Generator(device=DEV).manual_seed(3)
    T, V = s.t_max, 1003
    logits = 2 * torch.randn((s.B, T, V), generator=g, device=DEV)
    draft = logits[:, :T - 1].argmax(-1).to(torch.int32)
    ua, u = torch.rand((s.B, T - 1), generator=g, device=DEV), torch.rand(s.B, generator=g, device=DEV)
    lens = st4.seq.tolist()
    acc, tok = st4.accept(logits, draft, ua, u, temperature=0.5, top_p=0.9)
    torch.cuda.synchronize()
    want = [SU.verify(logits[b, :s.n_query[b]].double().cpu().numpy(), draft[b].tolist(), ua[b].cpu().numpy(), float(u[b]),
                      (0.5, 0, 0.9, 0.0)) for b in range(s.B)]
    assert list(zip(acc.tolist(), tok.tolist())) == want
    assert st4.seq.tolist() == [n + a for n, (a, _) in zip(lens, want)]
    if not paged:
        assert max(st4.seq.tolist()) > s.n_max  # (the step's calls are planned for lengths up to n_max)

    # eviction by accumulated attention, down to 200 positions; every cache and the weights follow one selection
    N = max(st4.seq.tolist())
    hist = torch.zeros((s.B, 1, N), device=DEV)
    D.score(est.q_target, score_k, st4.seq, list(range(s.num_q_heads)), init=hist, out=hist, max_len=N,
            page_table=four[0].page_table)
    old = [D.kv4_read(f.k, f.v, [0] * s.B, n_query=st4.seq, nq_max=N, page_table=f.page_table, max_len=0) for f in four]
    old_hist, old_draft, old_len = hist.clone(), [k.clone() for k in est.draft_k], st4.seq.tolist()
    idx, cnt = st4.evict(hist, 200)
    torch.cuda.synchronize()
    assert st4.seq.tolist() == [min(200, n) for n in old_len] == cnt.view(-1).tolist()
    new = [D.kv4_read(f.k, f.v, [0] * s.B, n_query=st4.seq, nq_max=200, page_table=f.page_table, max_len=0) for f in four]
    for b in range(s.B):
        at = idx[b, 0, :int(cnt[b, 0])].long()
        w = old_hist[b, 0, :old_len[b]]
        others = torch.ones(old_len[b], dtype=torch.bool, device=DEV)
        others[at] = False
        assert others[:4].sum() == 0 and others[-16:].sum() == 0
        assert w[others].max() <= w[at[4:-16]].min()
        for (k0, v0), (k1, v1) in zip(old, new):
            assert torch.equal(k1[b, :len(at)], k0[b, at]) and torch.equal(v1[b, :len(at)], v0[b, at])
        for k0, k1 in zip(old_draft, est.draft_k):
            assert torch.equal(k1[b, :len(at)], k0[b, at])
        assert torch.equal(hist[b, 0, :len(at)], old_hist[b, 0, at])

    # the next step, over what is left
    st4.run()
    torch.cuda.synchronize()
    n2 = st4.seq.tolist()
    for l, f in enumerate(four):
        k, v = D.kv4_read(f.k, f.v, [0] * s.B, n_query=[n + t for n, t in zip(n2, s.n_query)], nq_max=210,
                          page_table=f.page_table, max_len=0)
        gs = s.group_size
        for b in range(s.B):
            sel = st4.idx[b, 0, :int(st4.cnt[b, 0])].tolist()
            for h in range(s.num_kv_heads):
                pos = sel + list(range(n2[b], n2[b] + s.n_query[b]))
                q = f.q[b, :s.n_query[b], h * gs:(h + 1) * gs].double().cpu().numpy().reshape(-1, 128)
                ref, tol = U.attention(q, k[b, pos, h].double().cpu().numpy(), v[b, pos, h].double().cpu().numpy(),
                                       np.repeat(len(sel) + 1 + np.arange(s.n_query[b]), gs), 128 ** -0.5)
                got = st4.outs[l][b, :s.n_query[b], h * gs:(h + 1) * gs].double().cpu().numpy().reshape(-1, 128)
                assert (np.abs(got - ref) <= tol).all(), f"layer {l} sequence {b} head {h}"


def test_step_over_4_bits_as_a_graph():
    s, layers, est = build(True)
    windows = [S.window_kv(s, l) for l in layers]
    st = S.VerifyStep(s, [S.layer4(s, l) for l in layers], est, DEV, windows=windows, score_k=layers[0].k)
    st.run()
    torch.cuda.synchronize()
    ref = [o.clone() for o in st.outs]
    st.capture()
    for r in range(3):
        for o in st.outs:
            o.zero_()
        torch.cuda.synchronize()
        st.replay()
        torch.cuda.synchronize()
        for o, x in zip(st.outs, ref):
            for b, t in enumerate(s.n_query):
                assert torch.equal(o[b, :t].view(torch.int16), x[b, :t].view(torch.int16)), f"replay {r}"


def test_4_bit_layers_need_a_scoring_cache():
    s, layers, est = build(False)
    four = [S.layer4(s, l) for l in layers]
    with pytest.raises(ValueError, match="score_k"):
        S.VerifyStep(s, four, est, DEV, windows=[S.window_kv(s, l) for l in layers])


def test_per_layer_selection_over_4_bits():
    """The per-layer step selects by the draft model alone: the sets of the bf16 step, and the 4-bit attention over them."""
    s = W.config("qwen7b").replace(B=2, seq_lens=(2000, 700), n_query=(5, 5), budget=(256, 256), m=(118, 118),
                                   planted=(20,), layers=2, draft=W.DraftShape(layers=4))
    layers = [W.make_layer(s, l, DEV) for l in range(s.layers)]
    est = W.make_estimation(s, layers[0], DEV)
    four = [S.layer4(s, l) for l in layers]
    st16 = S.PerLayerSelectionStep(s, layers, est, DEV, n_target=8)
    st4 = S.PerLayerSelectionStep(s, four, est, DEV, n_target=8)
    st16.run()
    st4.run()
    torch.cuda.synchronize()
    B = s.B
    assert torch.equal(st4.cnt, st16.cnt)
    for r in range(4 * B):
        assert torch.equal(st4.idx[r, 0, :int(st4.cnt[r, 0])], st16.idx[r, 0, :int(st4.cnt[r, 0])])
    for i, L in enumerate(four):
        j = S.draft_layer_of(i, 8, 4)
        ref = D.sparse_verify_attn_kv4(L.q, L.k, L.v, st4.idx[j * B:(j + 1) * B], st4.cnt[j * B:(j + 1) * B], st4.seq)
        torch.cuda.synchronize()
        assert torch.equal(st4.outs[i].view(torch.int16), ref.view(torch.int16))
