"""One verification step of long-context speculative decoding on the GPU, planned once and
replayed: the target scoring-head score, the draft scores (accumulated over the draft
layers), the tiered top-k, and for every target layer the window's K/V append followed by
the sparse verification attention with the one index set (Sec. 3.2: a global, layer-invariant
selection; accepted tokens are appended to the cache).  Every launch is a prepared libdustin
call on one stream, so the whole step can be captured in a HIP graph and replayed.

The layers' caches may be held in 4 bits (layer4); the scoring layer's keys then stay in bf16 beside them.  After a step,
accept() verifies the drafted tokens against the target's logits and keeps the accepted ones, and evict() cuts every
cache to the positions with the most accumulated attention.
"""
import dataclasses
from typing import List, Optional

import torch

from . import (KV4, TOPK_MAX_LEN, digit_hist, kv4_append, kv4_empty, kv_evict, plan_kv4_append, plan_kv_append,
               plan_kv_commit, plan_score, plan_score_calls, plan_score_layers, plan_score_per_layer,
               plan_sparse_verify_attn, plan_sparse_verify_attn_kv4, plan_topk, topk, verify_tokens)


def window_kv(s, layer) -> tuple:
    """K and V of the verification window, [B, T_max, Hkv, d] each: the rows the layer's cache
    holds at [N_b, N_b + T_b) (what the target model's projections of the window tokens give)."""
    kk, vv = layer.contiguous_kv(s)
    B, T = s.B, s.t_max
    k_new = torch.zeros((B, T, s.num_kv_heads, s.head_dim), dtype=torch.bfloat16, device=kk.device)
    v_new = torch.zeros_like(k_new)
    for b in range(B):
        n, t = s.seq_lens[b], s.n_query[b]
        k_new[b, :t] = kk[b, n:n + t]
        v_new[b, :t] = vv[b, n:n + t]
    return k_new, v_new


def layer4(s, layer):
    """The layer with its caches in 4 bits: the rows that they hold, window included, appended to empty ones (in the
    same pages)."""
    kk, vv = layer.contiguous_kv(s)
    B, n, paged = layer.k.shape[0], layer.k.shape[1], layer.page_table is not None
    k, v = kv4_empty(B, n, s.num_kv_heads, s.head_dim, layer.k.device)
    rows = [x + y for x, y in zip(s.seq_lens, s.n_query)]
    T = max(rows)
    kv4_append(kk[:, :T], vv[:, :T], k, v, [0] * s.B, n_query=rows, page_table=layer.page_table,
               max_len=(layer.page_table.shape[1] * n if paged else n) - T)
    return dataclasses.replace(layer, k=k, v=v)


def _place(cache) -> int:
    """Where a cache lies: views of one cache are that cache."""
    return (cache.data if isinstance(cache, KV4) else cache).data_ptr()


def _plan_sparse(layer):
    """The sparse attention of the layer's kind of cache."""
    return plan_sparse_verify_attn_kv4 if isinstance(layer.k, KV4) else plan_sparse_verify_attn


class VerifyStep:
    """The step's launches over fixed buffers: run() enqueues them eagerly, capture() records
    them in a HIP graph and replay() launches the graph.  score_k: the scoring layer's keys in bf16, where the layers'
    caches are held in 4 bits (their rows follow those of the first layer).  The calls are planned for lengths of up to
    s.n_max before the window: once accepted tokens lead past it, evict() or plan a new step."""

    def __init__(self, s, layers, est, device, windows: Optional[list] = None, append: bool = True, score_k=None):
        self.s, self.layers, self.est, self.append = s, layers, est, append
        self.score_k = layers[0].k if score_k is None else score_k
        if isinstance(self.score_k, KV4):
            raise ValueError("the scores read a bf16 cache: with 4-bit layers, give score_k")
        if windows is None and isinstance(layers[0].k, KV4):
            raise ValueError("with 4-bit layers, give the windows' K and V")
        i32 = lambda x: torch.tensor(list(x), dtype=torch.int32, device=device)
        self.seq, self.nq, self.gam = i32(s.seq_lens), i32(s.n_query), i32(s.draft_gamma)
        self.bud, self.mm = i32(s.budget), i32(s.m)
        N = s.n_max
        self.s_t = torch.zeros((s.B, s.groups, N), dtype=torch.float32, device=device)
        self.s_d = torch.zeros((s.B, 1, N), dtype=torch.float32, device=device)
        self.idx = torch.zeros((s.B, s.groups, s.k_max), dtype=torch.int32, device=device)
        self.cnt = torch.zeros((s.B, s.groups), dtype=torch.int32, device=device)
        self.outs = [torch.empty_like(l.q) for l in layers]
        self.windows = windows if windows is not None else [window_kv(s, l) for l in layers]
        # with one selection group, the score calls count their outputs by top key digit and
        # the top-k takes those counts in place of its first pass over each row
        self.hist_t = digit_hist(s.B, device) if s.groups == 1 else None
        self.hist_d = digit_hist(s.B, device) if s.groups == 1 and est.s_draft_given is None else None
        self.graph = None
        self.ops = self._plan()

    def _plan(self, stream=None) -> List:
        """The step's operations, bound to `stream` (None: the current stream)."""
        s, est, N = self.s, self.est, self.s.n_max
        init = est.init_target
        if init is not None and s.groups > 1:  # one historical row, the same for every group
            init = init.expand(s.B, s.groups, N)
        target = plan_score(est.q_target, self.score_k, self.seq, s.target_heads, groups=s.groups,
                            init=init, out=self.s_t, max_len=N, page_table=self.layers[0].page_table,
                            stream=stream)
        if est.s_draft_given is not None:
            given = est.s_draft_given
            ops = [plan_score_calls([target], stream=stream, digit_hists=[self.hist_t]),
                   lambda: self.s_d.copy_(given)]
        else:
            # the target's and the draft's scores in one call (one launch where the library can)
            draft = plan_score_layers(est.draft_q, est.draft_k, self.seq, s.draft.heads, n_query=self.gam,
                                      out=self.s_d, max_len=N, stream=stream, ws_tag="score_draft")
            ops = [plan_score_calls([target, draft], stream=stream, digit_hists=[self.hist_t, self.hist_d])]
        ops.append(plan_topk(self.s_d, self.s_t, self.seq, s.k_max, budget=self.bud, m=self.mm,
                             n_sink=s.n_sink, n_window=s.n_window, groups=s.groups, idx=self.idx,
                             count=self.cnt, hist_d=self.hist_d, hist_t=self.hist_t, stream=stream))
        if self.append and _place(self.score_k) != _place(self.layers[0].k):
            ops.append(plan_kv_append(self.windows[0][0], None, self.score_k, None, self.seq, n_query=self.nq,
                                      page_table=self.layers[0].page_table, max_len=N, stream=stream))
        for L, o, (k_new, v_new) in zip(self.layers, self.outs, self.windows):
            if self.append:
                ops.append((plan_kv4_append if isinstance(L.k, KV4) else plan_kv_append)(
                    k_new, v_new, L.k, L.v, self.seq, n_query=self.nq, page_table=L.page_table, max_len=N,
                    stream=stream))
            bound = dict(max_len=N) if isinstance(L.k, KV4) else {}  # (the lengths that its append takes)
            ops.append(_plan_sparse(L)(L.q, L.k, L.v, self.idx, self.cnt, self.seq, n_query=self.nq,
                                       page_table=L.page_table, out=o, stream=stream, **bound))
        return ops

    def run(self):
        for op in self.ops:
            op()

    def capture(self):
        """Records the step in a HIP graph on a capture stream of its own.  The capture
        stream's workspaces are allocated (zeroed) by a planning pass before the capture
        starts, so nothing is allocated or cleared while recording."""
        self.run()
        cs = torch.cuda.Stream()
        self._plan(stream=cs)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=cs):
            ops = self._plan(stream=cs)
            for op in ops:
                op()
        self._graph_ops = ops  # keeps the marshalled arguments alive
        self._capture_stream = cs
        self.graph = g
        return g

    def replay(self):
        self.graph.replay()

    def commit(self, accepted: torch.Tensor):
        """After verification: N_b += accepted_b (clamped to [0, T_b])."""
        plan_kv_commit(self.seq, accepted, n_query=self.nq, nq_max=self.s.t_max)()

    def accept(self, logits, draft, u_accept, u, **kw):
        """The drafted tokens against the target's logits [B, T_max, V] of the window (verify_tokens, with its settings):
        keeps the accepted ones' rows; returns (accepted, token)."""
        accepted, token = verify_tokens(logits, draft, u_accept, u, n_query=self.nq, **kw)
        self.commit(accepted)
        return accepted, token

    def evict(self, weights: torch.Tensor, keep: int):
        """Cuts every cache, in place, to the keep positions of each sequence with the largest weights (fp32
        [B, 1, >= n_max], such as the accumulated target scores s_t), sinks and recent ones among them; the weights, the
        estimation's arrays over the positions (a history, given draft scores) and the lengths follow.  Behind the kept
        positions these arrays are zero: positions to come have no history.  Returns (idx, count)."""
        s, first = self.s, self.layers[0]
        # accepted tokens may lie past the weights' end: without a weight, but as positions (the most recent ones)
        missing = min(s.n_max + s.t_max, TOPK_MAX_LEN) - weights.shape[2]
        ranked = torch.nn.functional.pad(weights, (0, missing)) if missing > 0 else weights
        idx, cnt = topk(None, ranked, self.seq, keep, n_sink=s.n_sink, n_window=s.n_window)
        arrays = {x.data_ptr(): x for x in (weights, self.est.init_target, self.est.s_draft_given) if x is not None}
        for x in arrays.values():
            self._cut(x, idx, cnt)
        done = set()

        def once(k, v, page_table, **kw):  # (layers, the scores and a draft model may share caches)
            new = {_place(x): x for x in (k, v) if x is not None and _place(x) not in done}
            done.update(new)
            if new:
                kv_evict(*(*new.values(), None)[:2], idx, cnt, page_table=page_table, **kw)

        once(first.k, first.v, first.page_table, new_lens=self.seq)
        for L in self.layers[1:]:
            once(L.k, L.v, L.page_table)
        once(self.score_k, None, first.page_table)
        for k in self.est.draft_k:
            once(k, None, None)
        return idx, cnt

    @staticmethod
    def _cut(x, idx, cnt):
        """An array over the positions, fp32 [B, 1, N], follows the kept ones; zero behind them, and for positions past
        its end (tokens that were accepted since it was written)."""
        N = x.shape[2]
        kept = idx[:, :, :N]
        kv_evict(None, None, kept, cnt, weights=x)
        stays = torch.arange(N, device=x.device) < cnt.unsqueeze(2)
        stays[:, :, :kept.shape[2]] &= kept < N
        x.masked_fill_(~stays, 0.0)


def draft_layer_of(layer: int, n_target: int, n_draft: int) -> int:
    """The draft layer whose relevance selects the tokens of target layer `layer`: layers
    matched by depth, target layer l to draft layer floor(l * n_draft / n_target)."""
    return min(n_draft - 1, layer * n_draft // n_target)


class PerLayerSelectionStep:
    """The SpecAttn-style step the paper compares with (appendix on SpecAttn): token relevance
    from every head of every draft layer, one index set per draft layer (no aggregation
    across layers), each target layer attending with the set of its depth-matched draft
    layer.  Launches: the per-layer draft scores (one or two, as a rule), one top-k over (draft layer, sequence)
    rows, then per target layer the sparse attention.  est holds the draft model's layers
    (draft_q, draft_k); n_target is the target model's depth for the layer matching."""

    def __init__(self, s, layers, est, device, n_target: Optional[int] = None):
        self.s, self.layers, self.est = s, layers, est
        i32 = lambda x: torch.tensor(list(x), dtype=torch.int32, device=device)
        self.seq, self.nq, self.gam = i32(s.seq_lens), i32(s.n_query), i32(s.draft_gamma)
        self.bud = i32(s.budget)
        Ld, B, N = len(est.draft_q), s.B, s.n_max
        self.n_draft = Ld
        self.n_target = len(layers) if n_target is None else n_target
        # selection rows are (draft layer, sequence), layer-major: layer j's sets and counts
        # are the contiguous rows [j B, (j + 1) B)
        self.seq_rows, self.bud_rows = self.seq.repeat(Ld), self.bud.repeat(Ld)
        self.rel = torch.zeros((Ld, B, 1, N), dtype=torch.float32, device=device)
        self.idx = torch.zeros((Ld * B, 1, s.k_max), dtype=torch.int32, device=device)
        self.cnt = torch.zeros((Ld * B, 1), dtype=torch.int32, device=device)
        self.outs = [torch.empty_like(l.q) for l in layers]
        self.ops = self._plan()

    def _plan(self) -> List:
        s, est, N, B = self.s, self.est, self.s.n_max, self.s.B
        heads = list(range(s.draft.num_q_heads))
        ops = [plan_score_per_layer(est.draft_q, est.draft_k, self.seq, heads, n_query=self.gam,
                                    out=self.rel, max_len=N)]
        ops.append(plan_topk(self.rel.view(self.n_draft * B, 1, N), None, self.seq_rows, s.k_max,
                             budget=self.bud_rows, n_sink=s.n_sink, n_window=s.n_window,
                             idx=self.idx, count=self.cnt))
        for i, (L, o) in enumerate(zip(self.layers, self.outs)):
            j = draft_layer_of(i, self.n_target, self.n_draft)
            ops.append(_plan_sparse(L)(L.q, L.k, L.v, self.idx[j * B:(j + 1) * B],
                                       self.cnt[j * B:(j + 1) * B], self.seq, n_query=self.nq,
                                       page_table=L.page_table, out=o))
        return ops

    def run(self):
        for op in self.ops:
            op()
