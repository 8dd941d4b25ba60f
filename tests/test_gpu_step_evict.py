"""The verification step after an eviction: what it scores and selects by is what a step planned anew over the cut caches
and the cut arrays would."""
import pytest
import torch

import paper_2606_24957_amd as D
from paper_2606_24957_amd import step as S
from paper_2606_24957_amd import workloads as W

pytestmark = pytest.mark.gpu
DEV = "cuda"


def build(name):
    if name == "tiny":  # a history, and the draft scores given
        s = W.config("tiny").replace(B=2, seq_lens=(2000, 700), n_query=(5, 3), budget=(256, 200), m=(118, 90))
    elif name == "one":  # one sequence, one layer
        s = W.config("tiny")
    else:  # a history, three draft layers, two target layers
        s = W.config("qwen7b").replace(B=2, seq_lens=(2000, 700), n_query=(5, 5), budget=(256, 256), m=(118, 118),
                                       planted=(20,), layers=2)
    layers = [W.make_layer(s, l, DEV) for l in range(s.layers)]
    est = W.make_estimation(s, layers[0], DEV)
    assert est.init_target is not None
    return s, layers, est


def cut(x, idx, cnt):
    """Arrays over positions, cut by the definition: the kept entries in order, nothing behind them."""
    y = torch.zeros_like(x)
    for b in range(x.shape[0]):
        at = idx[b, 0, :int(cnt[b, 0])].long()
        inside = at < x.shape[2]
        y[b, 0, :len(at)][inside] = x[b, 0, at[inside]]
    return y


def anew(s, st, est_arrays, est):
    """A step planned over copies of what the evicted one holds, with the arrays given."""
    layers = [W.Layer(l.q, l.k.clone(), l.v.clone(), l.page_table) for l in st.layers]
    est2 = W.Estimation(est.q_target, est_arrays[0], est_arrays[1], est.draft_q, [k.clone() for k in est.draft_k])
    st2 = S.VerifyStep(s, layers, est2, DEV, windows=st.windows)
    st2.seq.copy_(st.seq)
    return st2


def same(s, a, b, lens):
    assert torch.equal(a.cnt, b.cnt)
    for i, n in enumerate(lens):
        c = int(a.cnt[i, 0])
        assert torch.equal(a.s_t[i, :, :n], b.s_t[i, :, :n]), f"sequence {i}: scores"
        assert torch.equal(a.s_d[i, :, :n], b.s_d[i, :, :n]), f"sequence {i}: draft scores"
        assert torch.equal(a.idx[i, 0, :c], b.idx[i, 0, :c]), f"sequence {i}: selection"
        for x, y in zip(a.outs, b.outs):
            assert torch.equal(x[i, :s.n_query[i]].view(torch.int16), y[i, :s.n_query[i]].view(torch.int16))


@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("by", ["scores", "history", "own"])
@pytest.mark.parametrize("name", ["tiny", "one", "history"])
def test_the_step_after_an_eviction(name, by, captured):
    s, layers, est = build(name)
    st = S.VerifyStep(s, layers, est, DEV)
    st.run()
    if captured:
        st.capture()
    torch.cuda.synchronize()
    weights = {"scores": st.s_t, "history": est.init_target, "own": torch.rand((s.B, 1, s.n_max + 9), device=DEV)}[by]
    old = [None if x is None else x.clone() for x in (est.init_target, est.s_draft_given, weights)]
    idx, cnt = st.evict(weights, 150)
    torch.cuda.synchronize()
    lens = [min(150, n) for n in s.seq_lens]
    assert st.seq.tolist() == lens
    want = [None if x is None else cut(x, idx, cnt) for x in old]
    for x, y in zip((est.init_target, est.s_draft_given, weights), want):
        assert (x is None) == (y is None)
        assert x is None or torch.equal(x, y)
    st2 = anew(s, st, want[:2], est)
    for _ in range(2):  # the next step, and the one after it with every token kept: new positions have no history
        st.replay() if captured else st.run()
        st2.run()
        torch.cuda.synchronize()
        same(s, st, st2, lens)
        for x in (st, st2):
            x.commit(x.nq)
        torch.cuda.synchronize()
        lens = [n + t for n, t in zip(lens, s.n_query)]
        assert st.seq.tolist() == lens


def test_tokens_accepted_past_the_weights_end_stay():
    """The step's scores end at its longest context; the tokens accepted after them are the most recent positions."""
    s, layers, est = build("history")
    st = S.VerifyStep(s, layers, est, DEV)
    st.run()
    st.commit(st.nq)
    torch.cuda.synchronize()
    keys = [l.k.clone() for l in layers]
    idx, cnt = st.evict(st.s_t, 150)
    torch.cuda.synchronize()
    assert cnt.view(-1).tolist() == st.seq.tolist() == [150, 150]
    for b, (n, t) in enumerate(zip(s.seq_lens, s.n_query)):
        recent = list(range(n + t - s.n_window, n + t))
        assert idx[b, 0, 150 - s.n_window:150].tolist() == recent
        for k, l in zip(keys, layers):
            assert torch.equal(l.k[b, 150 - s.n_window:150].view(torch.int16), k[b, recent].view(torch.int16))
        assert (st.s_t[b, 0, 150 - t:] == 0).all() or n < s.n_max  # (past the end: no weight yet)


def test_caches_that_share_memory_are_cut_once():
    """A second view of the scoring keys, a layer that has another's keys, a draft layer that reads a target layer's."""
    s, layers, est = build("history")
    two = [layers[0], W.Layer(layers[1].q, layers[0].k[:], layers[1].v)]
    draft = [est.draft_k[0], layers[0].k[:], est.draft_k[0].view(est.draft_k[0].shape)]
    shared = W.Estimation(est.q_target, est.init_target, None, est.draft_q, draft)
    st = S.VerifyStep(s.replace(draft=None), two, W.Estimation(est.q_target, est.init_target, torch.rand_like(est.init_target)),
                      DEV, windows=[S.window_kv(s, l) for l in layers], score_k=layers[0].k.view(layers[0].k.shape))
    st.est = shared
    held = [layers[0].k, layers[0].v, layers[1].v, draft[0]]
    old = [x.clone() for x in held]
    idx, cnt = st.evict(torch.rand((s.B, 1, s.n_max), device=DEV), 150)
    torch.cuda.synchronize()
    for x, y in zip(held, old):
        for b in range(s.B):
            at = idx[b, 0, :int(cnt[b, 0])].long()
            assert torch.equal(x[b, :len(at)].view(torch.int16), y[b, at].view(torch.int16))
            assert torch.equal(x[b, len(at):].view(torch.int16), y[b, len(at):].view(torch.int16))
    # and the scoring keys of a second view are not appended by themselves
    assert len(st.ops) == 2 + 1 + 2 * len(layers)


def test_weights_alone():
    """Arrays over the positions without a cache, to others and in place, several groups."""
    g = torch.Generator(device=DEV).manual_seed(1)
    B, G, N, K = 3, 4, 5000, 4001
    w = torch.rand((B, G, N), generator=g, device=DEV)
    idx = torch.sort(torch.rand((B, G, N), generator=g, device=DEV).argsort(-1)[:, :, :K]).values.int()
    cnt = torch.randint(0, K + 1, (B, G), generator=g, device=DEV).int()
    cnt[0, 0], cnt[1, 1] = 0, K
    lens = torch.full((B,), -1, dtype=torch.int32, device=DEV)
    out = torch.full((B, G, K), -1.0, device=DEV)
    want, inplace = out.clone(), w.clone()
    for b in range(B):
        for j in range(G):
            c = int(cnt[b, j])
            want[b, j, :c] = w[b, j, idx[b, j, :c].long()]
            inplace[b, j, :c] = want[b, j, :c]
    D.kv_evict(None, None, idx, cnt, weights=w, weights_out=out, new_lens=lens)
    torch.cuda.synchronize()
    assert torch.equal(out, want) and torch.equal(lens, cnt[:, 0])
    assert D.kv_evict(None, None, idx, cnt, weights=w) == (None, None)
    torch.cuda.synchronize()
    assert torch.equal(w, inplace)
    with pytest.raises(ValueError, match="only weights"):
        D.kv_evict(None, None, idx, cnt, new_lens=lens)
    with pytest.raises(ValueError, match="only weights"):
        D.kv_evict(None, None, idx, cnt, weights=w, k_out=out)


def test_weights_are_not_written_over_rows_still_to_be_read():
    w = torch.rand((2, 3, 500), device=DEV)
    idx = torch.arange(100, 140, dtype=torch.int32, device=DEV).expand(2, 3, 40).contiguous()
    cnt = torch.full((2, 3), 40, dtype=torch.int32, device=DEV)
    dense = w.view(-1)[:240].view(2, 3, 40)
    with pytest.raises(ValueError, match="another length"):
        D.kv_evict(None, None, idx, cnt, weights=w, weights_out=dense)
    with pytest.raises(ValueError, match="another length"):
        D.kv_evict(None, None, idx[:, :1], cnt[:, :1], weights=w[:, :1], weights_out=dense[:, :1])
    want = w[:, :, 100:140].clone()
    D.kv_evict(None, None, idx, cnt, weights=w, weights_out=w[:, :, :200])  # its own rows
    assert torch.equal(w[:, :, :40], want)
    D.kv_evict(None, None, idx[:1, :1], cnt[:1, :1], weights=w, weights_out=dense)  # one row
    torch.cuda.synchronize()


def test_sequences_of_one_cache_are_not_cut_in_place():
    k = torch.zeros((1, 64, 2, 128), dtype=torch.bfloat16, device=DEV)
    idx, cnt = torch.arange(8, 16, dtype=torch.int32, device=DEV).expand(3, 1, 8).contiguous(), torch.full((3, 1), 8, dtype=torch.int32, device=DEV)
    with pytest.raises(D.DustinError):
        D.kv_evict(k.expand(3, 64, 2, 128), None, idx, cnt)
    D.kv_evict(k.expand(3, 64, 2, 128), None, idx, cnt, k_out=torch.empty((3, 8, 2, 128), dtype=torch.bfloat16, device=DEV))
    torch.cuda.synchronize()


@pytest.mark.parametrize("preset", ["qwen7b", "ragged"])
def test_a_step_over_4_bits_takes_one_length_in_all_its_calls(preset):
    """Lengths past the planned ones (the caller's to avoid) are clamped alike by append and attention: the window that
    the one writes is the window that the other reads."""
    s = W.config(preset)
    s = s.replace(B=2, seq_lens=(700, 300), n_query=(5, 3), budget=(128, 100), m=(54, 40), planted=(20, 20), layers=1)
    layer = W.make_layer(s, 0, DEV)
    est = W.make_estimation(s, layer, DEV)
    four = S.layer4(s, layer)
    st = S.VerifyStep(s, [four], est, DEV, windows=[S.window_kv(s, layer)], score_k=layer.k)
    st.run()
    torch.cuda.synchronize()
    want = st.outs[0].clone()
    st.seq[0] += 2
    st.run()
    torch.cuda.synchronize()
    for b, t in enumerate(s.n_query):
        assert torch.equal(st.outs[0][b, :t].view(torch.int16), want[b, :t].view(torch.int16))
