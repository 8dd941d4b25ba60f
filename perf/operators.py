"""The operators around sparse verification that a serving loop with a compressed cache runs, as measurable cases.

A case names one of them, at a model shape, batch, context length, speculative depth, budget or vocabulary:

    append     the window's (or a prompt's) K and V rows into a cache held in 4 bits, and the same rows read back as
               the values the cache now stands for
    sparse     one target layer's verification attention over a selected set of a 4-bit cache
    dense      the same over the whole 4-bit cache
    evict      one layer's kept rows (chosen by accumulated attention weight) into a shorter cache, with the weights
               and the new lengths
    sample     next tokens from logits with temperature, top-k, top-p and min-p, from given random numbers (and, for
               a draft model, the distribution that they were drawn from)
    verify     the drafted tokens of a verification window accepted or rejected against the target's logits, and the
               token that follows

A 4-bit cache holds a row of d channels as d / 32 blocks: elements in E2M1 (1 sign, 2 exponent, 1 mantissa bit: 0, 0.5,
1, 1.5, 2, 3, 4, 6), two to a byte, the even channel in the low half, and one byte e for each block, a scale of 2^(e - 127).

The shapes are those of the workload presets: 8 query heads over 1 KV head, 28 over 4 and 64 over 8, of 128 channels.
"""
import math
import random

import numpy as np
import torch

own = False  # False: the plain forms; True: the framework's operators

D, PAGE, SINK, WINDOW = 128, 16, 4, 16
HKV = {8: 1, 28: 4, 64: 8}  # query heads: KV heads
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
CUT = 2.0 ** -45  # a token's weight below this part of the largest counts as zero


def _attn(name, kind, B, Hq, N, T, k, *, paged=False, ragged=0):
    c = dict(kind=kind, B=B, Hq=Hq, N=N, T=T, k=k, paged=paged, ragged=ragged)
    return dict(c, name=name) if name else c


def _append(name, B, Hq, N, T, *, paged=False, ragged=0):
    return _attn(name, "append", B, Hq, N, T, 0, paged=paged, ragged=ragged)


def _evict(name, B, Hq, N, k, *, four=False, paged=False, ragged=0):
    c = dict(_attn(None, "evict", B, Hq, N, 0, k, paged=paged, ragged=ragged), four=four)
    return dict(c, name=name) if name else c


def _sample(name, rows, V, *, dtype="bf16", probs=False, filters="mixed"):
    c = dict(kind="sample", rows=rows, V=V, dtype=dtype, probs=probs, filters=filters)
    return dict(c, name=name) if name else c


def _verify(name, B, T, V, *, dtype="bf16", drawn=True, filters="mixed", ragged=0):
    c = dict(kind="verify", B=B, T=T, V=V, dtype=dtype, drawn=drawn, filters=filters, ragged=ragged)
    return dict(c, name=name) if name else c


def listed():
    return [
        # a serving batch's verification window into its paged cache, before each layer's attention
        _append("append_window", 16, 64, 32768, 5, paged=True, ragged=11),
        # prompts of a small batch into an empty cache
        _append("append_prompt", 4, 28, 0, 8192),
        # one layer of a small model, one sequence: a call's latency is all there is
        _attn("sparse_tiny", "sparse", 1, 8, 2048, 5, 256),
        # one of the 80 layers of a full serving batch, 32K contexts
        _attn("sparse_72b", "sparse", 16, 64, 32768, 5, 2048),
        # single tokens over the whole cache, the smaller model
        _attn("dense_7b", "dense", 4, 28, 8192, 1, 0),
        # the full cache at continuous batching: paged, contexts of 4K to 65K, a depth per sequence
        _attn("dense_ragged", "dense", 16, 64, 65536, 9, 0, paged=True, ragged=4000),
        # one user's long context cut to the budget
        _evict("evict_one", 1, 64, 32768, 8192),
        # a serving batch's 4-bit pages into fresh ones
        _evict("evict_pages", 16, 64, 32768, 4096, four=True, paged=True, ragged=17),
        # a draft model's next token for one user, and the distribution that it was drawn from
        _sample("sample_one", 1, 32000, dtype="fp32", probs=True),
        # requests of a large decoding batch with settings of their own
        _sample("sample_batch", 128, 151936),
        # one user's window, drafted greedily
        _verify("verify_one", 1, 5, 151936, drawn=False),
        # a serving batch's windows against the distributions that the drafts were drawn from
        _verify("verify_batch", 16, 5, 151936, ragged=23),
    ]


def draw(rng: random.Random):
    """A case of the same ranges: any operator and model, sizes spread over their logarithm."""

    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    most = {}
    for c in listed():
        most[c["kind"]] = max(most.get(c["kind"], 0), work(c)["bytes"])
    while True:
        kind = rng.choice(("append", "sparse", "sparse", "dense", "evict", "sample", "sample", "verify"))
        Hq, B = rng.choice((8, 28, 64, 64)), log_int(1, 16)
        paged = rng.random() < 0.5
        ragged = rng.randint(1, 9999) if B > 1 and rng.random() < 0.6 else 0
        if kind == "append":
            c = _append(None, B, Hq, rng.choice((0, log_int(1, 32768))), log_int(1, 8192), paged=paged, ragged=ragged)
        elif kind == "sparse":
            N = log_int(64, 65536)
            c = _attn(None, kind, B, Hq, N, rng.randint(1, 9), min(log_int(24, 4096), N), paged=paged, ragged=ragged)
        elif kind == "dense":
            c = _attn(None, kind, B, Hq, log_int(1, 65536), rng.randint(1, 9), 0, paged=paged, ragged=ragged)
        elif kind == "evict":
            N = log_int(64, 32768)
            c = _evict(None, B, Hq, N, max(21, min(log_int(32, 16384), N - N // 8)), four=rng.random() < 0.5,
                       paged=paged, ragged=ragged)
        else:
            V, dtype = log_int(1000, 151936), rng.choice(("bf16", "bf16", "fp32"))
            filters = rng.choice(("mixed", "mixed", "none", "top_k", "top_p"))
            if kind == "sample":
                c = _sample(None, log_int(1, 128), V, dtype=dtype, probs=rng.random() < 0.4, filters=filters)
            else:
                c = _verify(None, B, rng.randint(1, 9), V, dtype=dtype, drawn=rng.random() < 0.7, filters=filters,
                            ragged=ragged)
        if work(c)["bytes"] <= most[kind]:
            return c


# ------------------------------------------------------------------- sizes of a case

def _sizes(c):
    """Per sequence: context, new or verified tokens, budget."""
    B, N, T, k = c["B"], c["N"], c["T"], c["k"]
    if not c["ragged"]:
        return [N] * B, [T] * B, [min(k, N)] * B
    g = random.Random(c["ragged"])
    n = [g.randint(N // 16, N) for _ in range(B)]
    return n, [g.randint((T + 2) // 3, T) for _ in range(B)], [min(x, max(21, x * k // max(N, 1))) for x in n]


def work(case):
    c, kind = case, case["kind"]
    if kind in ("sample", "verify"):
        size = 2 if c["dtype"] == "bf16" else 4
        if kind == "sample":
            n = c["rows"] * c["V"]
            return {"bytes": n * size + (4 * n if c["probs"] else 0) + 8 * c["rows"], "flops": 3 * n}
        rows = sum(_windows(c))
        return {"bytes": rows * c["V"] * size + (4 * c["B"] * c["V"] if c["drawn"] and c["T"] > 1 else 0),
                "flops": 3 * rows * c["V"]}
    n, t, k = _sizes(c)
    h, row4, row16 = HKV[c["Hq"]], 2 * (D // 2 + D // 32), 4 * D  # bytes of a K and a V row
    if kind == "append":
        return {"bytes": sum(t) * h * (2 * row16 + 2 * row4), "flops": 4 * sum(t) * h * D}
    if kind == "evict":
        row = row4 if c["four"] else row16
        extra = (row4 + row16) * h if c["four"] else 0  # the kept rows read back as values
        return {"bytes": sum(k) * (2 * h * row + extra + 12), "flops": 0}
    seen = k if kind == "sparse" else n
    byts = sum(h * row4 * (x + y) + 4 * y * c["Hq"] * D + (4 * x if kind == "sparse" else 0) for x, y in zip(seen, t))
    return {"bytes": byts, "flops": sum(4 * c["Hq"] * D * y * (x + (y + 1) / 2) for x, y in zip(seen, t))}


def _windows(c):
    if not c["ragged"]:
        return [c["T"]] * c["B"]
    g = random.Random(c["ragged"])
    return [g.randint((c["T"] + 2) // 3, c["T"]) for _ in range(c["B"])]


# ------------------------------------------------------------------- the 4-bit format

def _to_codes(x):
    """bf16 rows [..., d] as packed codes uint8 [..., d / 2] and block scales uint8 [..., d / 32]."""
    y = torch.nan_to_num(x.float(), nan=0.0, posinf=3.3895313892515355e38, neginf=-3.3895313892515355e38)
    y = y.unflatten(-1, (-1, 32))
    e = (torch.frexp(y.abs().amax(-1))[1] - 3).clamp_min(-125)
    y = torch.ldexp(y, -e[..., None])
    a = y.abs().clamp_max(6.0)
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    r = torch.round(a / step) * step
    code = torch.where(r < 2, 2 * r, torch.where(r < 4, r + 2, r / 2 + 4)).to(torch.uint8)
    code = (code + 8 * torch.signbit(y).to(torch.uint8)).flatten(-2)
    return code[..., 0::2] | (code[..., 1::2] << 4), (e + 127).to(torch.uint8)


def _values(data, scales):
    """The values of packed rows, fp32 (every one of them a bf16 number)."""
    grid = torch.tensor(GRID + tuple(-g for g in GRID), dtype=torch.float32, device=data.device)
    v = torch.stack((grid[(data & 15).long()], grid[(data >> 4).long()]), -1).flatten(-2)
    s = torch.ldexp(torch.ones((), device=data.device), scales.int() - 127)
    return (v.unflatten(-1, (-1, 32)) * s[..., None]).flatten(-2)


# ------------------------------------------------------------------- inputs

def _i32(x, dev):
    return torch.tensor(list(x), dtype=torch.int32, device=dev)


def _pages(need, g, dev):
    """A page table whose rows are consecutive runs of a permutation of the pool, and the pool's size."""
    per = [max(1, -(-x // PAGE)) for x in need]
    perm = torch.randperm(sum(per), generator=g, device=dev).to(torch.int32)
    pt = torch.zeros((len(per), max(per)), dtype=torch.int32, device=dev)
    at = 0
    for b, p in enumerate(per):
        pt[b, :p] = perm[at:at + p]
        at += p
    return pt, sum(per)


def _rows_of(pt, b, pos):
    """Where positions `pos` of sequence b lie: two indexes into a cache's first two axes."""
    if pt is None:
        return torch.full_like(pos, b), pos
    return pt[b].long()[pos // PAGE], pos % PAGE


def _kept(n, k, g, dev):
    """k of n positions in ascending order: the sinks, the recent ones, and others at random."""
    if k >= n:
        return torch.arange(n, device=dev)
    w = torch.rand(n, generator=g, device=dev)
    w[:SINK] = 2.0
    w[max(0, n - WINDOW):] = 2.0
    return torch.sort(torch.topk(w, k).indices).values


def _selection(n, k, g, dev):
    kmax = max(1, max(k))
    idx = torch.zeros((len(n), 1, kmax), dtype=torch.int32, device=dev)
    for b, (x, y) in enumerate(zip(n, k)):
        idx[b, 0, :y] = _kept(x, y, g, dev).to(torch.int32)
    return idx, _i32(k, dev).view(-1, 1)


def _cache4(rows, cap, h, pt, pool, dev):
    shape = (len(rows), cap, h) if pt is None else (pool, PAGE, h)
    return (torch.zeros(shape + (2, D // 2), dtype=torch.uint8, device=dev),
            torch.zeros(shape + (2, D // 32), dtype=torch.uint8, device=dev))


def _fill4(data, scales, need, h, pt, g, dev):
    for b, n in enumerate(need):
        if n:
            kv = torch.randn((n, h, 2, D), generator=g, device=dev, dtype=torch.bfloat16)
            kv[..., 0, :] *= 1.0 + 3.0 * (torch.arange(D, device=dev) % 37 == 5)  # keys have strong channels
            where = _rows_of(pt, b, torch.arange(n, device=dev))
            data[where], scales[where] = _to_codes(kv)


def _settings(n, filters, g, dev):
    """Temperature, top-k, top-p and min-p of n requests."""
    pick = lambda xs: torch.tensor(xs, device=dev)[torch.randint(len(xs), (n,), generator=g, device=dev)]
    off = filters in ("none", "top_k", "top_p")
    t = pick((0.7, 1.0)) if off else pick((0.0, 0.6, 0.7, 0.8, 1.0, 1.0))
    k = pick((20, 40, 50)) if filters == "top_k" else pick((0,)) if off else pick((0, 0, 20, 50))
    p = pick((0.8, 0.9, 0.95)) if filters == "top_p" else pick((1.0,)) if off else pick((1.0, 0.8, 0.9, 0.95))
    m = pick((0.0,)) if off else pick((0.0, 0.0, 0.05))
    return t.float(), k.to(torch.int32), p.float(), m.float()


def _logits(rows, V, g, dev):
    """A wide bulk and, in every row, a few tokens far above it."""
    x = 2.0 * torch.randn((rows, V), generator=g, device=dev)
    at = torch.randint(V, (rows, 24), generator=g, device=dev)
    up = 7.0 + 7.0 * torch.rand((rows, 24), generator=g, device=dev)
    return x.scatter_(1, at, up)


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(int(seed) & 0x7FFFFFFF)
    c, kind = case, case["kind"]
    st = dict(case=case, dev=dev)
    if kind in ("sample", "verify"):
        dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
        B, T = (c["rows"], 1) if kind == "sample" else (c["B"], c["T"])
        st["set"] = _settings(B, c["filters"], g, dev)
        base = _logits(B * T, c["V"], g, dev)
        st["logits"] = base.to(dt) if kind == "sample" else base.to(dt).view(B, T, c["V"])
        st["u"] = torch.rand(B, generator=g, device=dev)
        if kind == "verify":
            st["nq"] = _i32(_windows(c), dev)
            st["ua"] = torch.rand((B, T - 1), generator=g, device=dev)
            near = base + 0.5 * torch.randn(base.shape, generator=g, device=dev)
            near = near.view(B, T, c["V"])[:, :T - 1]
            if c["drawn"]:
                # the draft model samples with the request's temperature (greedy ones: nearly so) from its 200 best
                t = st["set"][0].clamp_min(0.05).view(B, 1, 1)
                best = torch.topk(near / t, min(200, c["V"]))
                q = torch.zeros_like(near).scatter_(2, best.indices, torch.softmax(best.values, -1))
                st["q"] = q.contiguous()
                at = torch.multinomial(q.reshape(-1, c["V"]), 1, generator=g) if T > 1 else torch.zeros((0, 1), device=dev)
                st["draft"] = at.view(B, T - 1).to(torch.int32)
            else:
                st["q"], st["draft"] = None, near.argmax(-1).to(torch.int32)
        if own:
            import paper_2606_24957_amd as da
            t, k, p, m = st["set"]
            kw = dict(temperature=t, top_k=k, top_p=p, min_p=m)
            if kind == "sample":
                probs = torch.empty((B, c["V"]), dtype=torch.float32, device=dev) if c["probs"] else None
                st["call"] = da.plan_sample(st["logits"], st["u"], probs=probs, **kw)
            else:
                st["call"] = da.plan_verify_tokens(st["logits"], st["draft"], st["ua"], st["u"], draft_probs=st["q"],
                                                   n_query=st["nq"], **kw)
        return st

    n, t, k = _sizes(c)
    h, tmax, four = HKV[c["Hq"]], max(t), kind != "evict" or c["four"]
    need = [x + y for x, y in zip(n, t)]
    pt, pool = _pages(need, g, dev) if c["paged"] else (None, 0)
    cap = max(1, max(need))
    st.update(n=n, t=t, k=k, h=h, pt=pt, seq=_i32(n, dev), nq=_i32(t, dev), max_len=max(n))
    if four:
        st["kv"] = _cache4(n, cap, h, pt, pool, dev)
        _fill4(*st["kv"], n if kind == "append" else need, h, pt, g, dev)
    else:
        shape = (c["B"], cap, h, 2, D) if pt is None else (pool, PAGE, h, 2, D)
        st["kv"] = (torch.randn(shape, generator=g, device=dev, dtype=torch.bfloat16),)
    if kind == "append":
        st["new"] = torch.randn((c["B"], tmax, 2, h, D), generator=g, device=dev, dtype=torch.bfloat16)
        st["out"] = torch.zeros((2, c["B"], tmax, h, D), dtype=torch.bfloat16, device=dev)
    elif kind == "evict":
        st["idx"], st["cnt"] = _selection(n, k, g, dev)
        kmax = st["idx"].shape[2]
        st["opt"], opool = _pages(k, g, dev) if c["paged"] else (None, 0)
        st["wts"] = torch.rand((c["B"], 1, max(n)), generator=g, device=dev).square()
        st["wout"] = torch.zeros((c["B"], 1, kmax), device=dev)
        st["lens"] = torch.zeros(c["B"], dtype=torch.int32, device=dev)
        if four:
            st["kvout"] = _cache4(n, kmax, h, st["opt"], opool, dev)
            st["out"] = torch.zeros((2, c["B"], kmax, h, D), dtype=torch.bfloat16, device=dev)
        else:
            shape = (c["B"], kmax, h, 2, D) if pt is None else (opool, PAGE, h, 2, D)
            st["kvout"] = (torch.zeros(shape, dtype=torch.bfloat16, device=dev),)
    else:
        st["q"] = 2.0 * torch.randn((c["B"], tmax, c["Hq"], D), generator=g, device=dev, dtype=torch.bfloat16)
        st["out"] = torch.zeros_like(st["q"])
        if kind == "sparse":
            st["idx"], st["cnt"] = _selection(n, k, g, dev)
    if own:
        st["calls"] = _plan(st, kind, four, tmax)
    return st


def _plan(st, kind, four, tmax):
    import paper_2606_24957_amd as da

    def half(kv, i):
        return da.KV4(kv[0][..., i, :], kv[1][..., i, :]) if four else kv[0][..., i, :]

    k, v = half(st["kv"], 0), half(st["kv"], 1)
    kw = dict(page_table=st["pt"])
    if kind == "append":
        kw.update(n_query=st["nq"], max_len=st["max_len"])
        return [da.plan_kv4_append(st["new"][:, :, 0], st["new"][:, :, 1], k, v, st["seq"], **kw),
                da.plan_kv4_read(k, v, st["seq"], k_out=st["out"][0], v_out=st["out"][1], **kw)]
    if kind == "evict":
        ko, vo = half(st["kvout"], 0), half(st["kvout"], 1)
        calls = [da.plan_kv_evict(k, v, st["idx"], st["cnt"], k_out=ko, v_out=vo, weights=st["wts"],
                                  weights_out=st["wout"], new_lens=st["lens"], out_page_table=st["opt"], **kw)]
        if four:
            calls.append(da.plan_kv4_read(ko, vo, torch.zeros_like(st["lens"]), n_query=st["cnt"].view(-1),
                                          page_table=st["opt"], max_len=0, k_out=st["out"][0], v_out=st["out"][1]))
        return calls
    kw.update(n_query=st["nq"], out=st["out"], max_len=st["max_len"])
    if kind == "sparse":
        return [da.plan_sparse_verify_attn_kv4(st["q"], k, v, st["idx"], st["cnt"], st["seq"], **kw)]
    return [da.plan_dense_verify_attn_kv4(st["q"], k, v, st["seq"], **kw)]


# ------------------------------------------------------------------- one pass

def run(state):
    st = state
    kind = st["case"]["kind"]
    if own:
        if kind in ("sample", "verify"):
            return st["call"]()
        for call in st["calls"]:
            call()
    elif kind == "sample":
        return _plain_sample(st["logits"], st["u"], st["set"], st["case"]["probs"])
    elif kind == "verify":
        return _plain_verify(st)
    elif kind == "append":
        _plain_append(st)
    elif kind == "evict":
        _plain_evict(st)
    else:
        _plain_attention(st, kind == "sparse")
    if kind != "evict":
        return st["out"]
    if st["case"]["four"]:
        return st["out"], st["wout"], st["lens"]
    return st["kvout"][0], st["wout"], st["lens"]


def _plain_append(st):
    data, scales = st["kv"]
    for b, (n, t) in enumerate(zip(st["n"], st["t"])):
        where = _rows_of(st["pt"], b, torch.arange(n, n + t, device=st["dev"]))
        data[where], scales[where] = _to_codes(st["new"][b, :t].transpose(1, 2))
        st["out"][:, b, :t] = _values(data[where], scales[where]).permute(2, 0, 1, 3).to(torch.bfloat16)


def _plain_evict(st):
    for b, k in enumerate(st["k"]):
        pos = st["idx"][b, 0, :k].long()
        src = _rows_of(st["pt"], b, pos)
        dst = _rows_of(st["opt"], b, torch.arange(k, device=st["dev"]))
        for a, o in zip(st["kv"], st["kvout"]):
            o[dst] = a[src]
        st["wout"][b, 0, :k] = st["wts"][b, 0][pos]
        if st["case"]["four"]:
            rows = _values(*(o[dst] for o in st["kvout"]))
            st["out"][:, b, :k] = rows.permute(2, 0, 1, 3).to(torch.bfloat16)
    st["lens"].copy_(st["cnt"].view(-1))


def _plain_attention(st, sparse):
    data, scales = st["kv"]
    h, dev, hq = st["h"], st["dev"], st["case"]["Hq"]
    for b, (n, t) in enumerate(zip(st["n"], st["t"])):
        pos = torch.arange(n + t, device=dev)
        if sparse:
            pos = torch.cat((st["idx"][b, 0, :st["k"][b]].long(), pos[n:]))
        where = _rows_of(st["pt"], b, pos)
        kv = _values(data[where], scales[where])
        q = st["q"][b, :t].float().view(t, h, hq // h, D).transpose(0, 1).reshape(h, -1, D)
        s = torch.matmul(q, kv[:, :, 0].permute(1, 2, 0).contiguous()) / math.sqrt(D)
        s = s.view(h, t, hq // h, -1)
        late = pos[None, :] > n + torch.arange(t, device=dev)[:, None]
        s = s.masked_fill(late[None, :, None, :], float("-inf"))
        p = torch.exp(s - s.amax(-1, keepdim=True))
        p = p / p.sum(-1, keepdim=True)
        o = torch.matmul(p.view(h, -1, pos.numel()), kv[:, :, 1].transpose(0, 1).contiguous())
        st["out"][b, :t] = o.view(h, t, hq // h, D).transpose(0, 1).reshape(t, hq, D).to(torch.bfloat16)


def _plain_weights(x, settings):
    """Weights [R, V] (fp64, the largest 1) of the tokens that each row's settings keep, the others 0."""
    t, k, p, m = (z[:, None] for z in settings)
    x, R, V = x.double(), x.shape[0], x.shape[1]
    x = torch.where(torch.isnan(x), -torch.inf, x)
    top = x.amax(-1, keepdim=True)
    order = torch.sort(x, dim=-1, descending=True, stable=True).indices
    w = torch.where(x == top, 1.0, torch.exp((x - top) / t.double()))
    w = torch.where((w < CUT) | (x == -torch.inf), 0.0, w)
    s = w.gather(1, order)
    rank = torch.arange(V, device=x.device)[None]
    s = torch.where((rank >= k) & (k > 0), 0.0, s)
    before = s.cumsum(-1) - s
    s = torch.where((before >= p.double() * s.sum(-1, keepdim=True)) & (p < 1) & (rank > 0), 0.0, s)
    s = torch.where(s >= m.double(), s, 0.0)
    s = torch.where((t > 0) | (rank == 0), s, 0.0)
    return torch.zeros_like(w).scatter_(1, order, s)


def _pick(w, u):
    """The first index whose running sum of w [R, V] passes u of the whole."""
    c = w.cumsum(-1)
    at = (c <= u.double()[:, None] * c[:, -1:]).sum(-1)
    last = w.shape[1] - 1 - (w > 0).flip(-1).to(torch.uint8).argmax(-1)
    return torch.where(c[:, -1] > 0, torch.minimum(at, last), -1).to(torch.int32)


def _plain_sample(x, u, settings, probs):
    w = _plain_weights(x, settings)
    token = _pick(w, u)
    return (token, (w / w.sum(-1, keepdim=True).clamp_min(1e-300)).float()) if probs else token


def _plain_verify(st):
    x, draft, q = st["logits"], st["draft"].long(), st["q"]
    B, T, V = x.shape
    w = _plain_weights(x.reshape(B * T, V), [z.repeat_interleave(T) for z in st["set"]])
    p = (w / w.sum(-1, keepdim=True).clamp_min(1e-300)).view(B, T, V)
    rows, nq = torch.arange(B, device=x.device), st["nq"].long()
    kept = torch.zeros(B, dtype=torch.long, device=x.device)
    for t in range(T - 1):
        px = p[rows, t, draft[:, t]]
        qx = q[rows, t, draft[:, t]].double() if q is not None else torch.ones_like(px)
        ok = (st["ua"][:, t].double() * qx < px) & (t < nq - 1) & (kept == t)
        kept += ok.long()
    last = p[rows, kept]
    if T > 1:
        at = kept.clamp_max(T - 2)
        if q is None:
            sub = torch.zeros_like(last).scatter_(1, draft[rows, at][:, None], 1.0)
        else:
            sub = q[rows, at].double()
        rest = torch.where((kept < nq - 1)[:, None], (last - sub).clamp_min(0), last)
        last = torch.where((rest.sum(-1) > 0)[:, None], rest, last)
    return torch.where(nq > 0, kept + 1, 0).to(torch.int32), _pick(last, st["u"])


# ------------------------------------------------------------------- from the definitions, in 64 bits

def _decode64(data, scales):
    """Row values by the format's arithmetic: (1 + m / 2) 2^(x - 1), or m / 2 where the exponent bits are zero."""
    c = torch.stack((data % 16, data // 16), -1).flatten(-2).to(torch.float64)
    sign = torch.where(c >= 8, -1.0, 1.0).double()
    c = c % 8
    x, m = torch.floor(c / 2), c % 2
    mag = torch.where(x > 0, (1 + m / 2) * torch.exp2(x - 1), m / 2)
    e = scales.to(torch.float64).repeat_interleave(32, dim=-1) - 127
    return sign * mag * torch.exp2(e)


def _round64(x):
    """Rows rounded into the format: the nearest of the signed grid, the even code where two are as near."""
    x = x.double()
    grid = torch.tensor(GRID, dtype=torch.float64, device=x.device)
    out = torch.empty_like(x)
    for i in range(0, x.shape[-1], 32):
        y = x[..., i:i + 32]
        big = y.abs().amax(-1, keepdim=True)
        e = torch.where(big > 0, torch.floor(torch.log2(big.clamp_min(1e-300))) - 2, -125.0).clamp_min(-125)
        a = y.abs() / torch.exp2(e)
        best = torch.zeros_like(a)
        for j in range(1, 8):  # the border between grid[j - 1] and grid[j]; on it, the even code
            edge = (grid[j - 1] + grid[j]) / 2
            best = torch.where((a >= edge) if j % 2 == 0 else (a > edge), grid[j], best)
        out[..., i:i + 32] = torch.sign(y) * best * torch.exp2(e)
    return out


def _exact_attention(st, sparse):
    data, scales = st["kv"]
    c, pt = st["case"], st["pt"]
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device=st["dev"])
    gs = c["Hq"] // st["h"]
    for b in range(c["B"]):
        n, t = st["n"][b], st["t"][b]
        pos = list(range(n + t)) if not sparse else st["idx"][b, 0, :st["k"][b]].tolist() + list(range(n, n + t))
        pos = torch.tensor(pos, device=st["dev"])
        if pt is None:
            rows, sc = data[b][pos], scales[b][pos]
        else:
            page = pt[b][torch.div(pos, PAGE, rounding_mode="floor")].long()
            rows, sc = data[page, pos % PAGE], scales[page, pos % PAGE]
        for g in range(st["h"]):
            kk, vv = (_decode64(rows[:, g, i], sc[:, g, i]) for i in (0, 1))
            for y in range(t):
                see = pos <= n + y
                s = (st["q"][b, y, g * gs:(g + 1) * gs].double() @ kk.T) / math.sqrt(D)
                s = torch.where(see[None], s, -torch.inf)
                out[b, y, g * gs:(g + 1) * gs] = torch.softmax(s, -1) @ vv
    return out


def _exact_kept(x, t, k, p, m):
    """One row (numpy, fp64): the weights of the kept tokens, others 0."""
    x = np.where(np.isnan(x), -np.inf, x.astype(np.float64))
    order = np.lexsort((np.arange(x.size), -x))
    top = x[order[0]]
    if top == -np.inf:
        return np.zeros(x.size)
    if not t > 0:
        w = np.zeros(x.size)
        w[order[0]] = 1.0
        return w
    with np.errstate(invalid="ignore"):
        w = np.where(x == top, 1.0, np.exp((x - top) / np.float64(t)))
    w[w < CUT] = 0.0
    n = min(k, x.size) if k > 0 else x.size
    if p < 1:
        run = np.cumsum(w[order[:n]])
        n = min(n, 1 + int(np.searchsorted(run, np.float64(p) * run[-1], side="left")))
    keep = np.zeros(x.size, dtype=bool)
    keep[order[:max(n, 1)]] = True
    return np.where(keep & (w >= m), w, 0.0)


def _exact_pick(w, u):
    if not (w > 0).any():
        return -1
    run = np.cumsum(w)
    return min(int(np.searchsorted(run, float(u) * run[-1], side="right")), int(np.flatnonzero(w)[-1]))


def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    c, kind, dev = case, case["kind"], st["dev"]
    if kind in ("sparse", "dense"):
        if work(case)["flops"] > 4e11:
            return None  # about 20 seconds and more
        return _exact_attention(st, kind == "sparse")
    if kind == "append":
        out = torch.zeros(st["out"].shape, dtype=torch.float64, device=dev)
        for b, t in enumerate(st["t"]):
            out[0, b, :t], out[1, b, :t] = _round64(st["new"][b, :t, 0]), _round64(st["new"][b, :t, 1])
        return out
    if kind == "evict":
        rows = []
        if not c["four"]:
            rows = torch.zeros(st["kvout"][0].shape, dtype=torch.float64, device=dev)
        else:
            rows = torch.zeros(st["out"].shape, dtype=torch.float64, device=dev)
        wts = torch.zeros(st["wout"].shape, dtype=torch.float64, device=dev)
        for b, k in enumerate(st["k"]):
            i = torch.arange(k, device=dev)
            pos = st["idx"][b, 0, :k].long()
            wts[b, 0, :k] = st["wts"][b, 0, pos]
            if st["pt"] is None:
                got = [a[b].index_select(0, pos) for a in st["kv"]]
            else:
                flat = st["pt"][b, pos // PAGE].long() * PAGE + pos % PAGE
                got = [a.flatten(0, 1).index_select(0, flat) for a in st["kv"]]
            if c["four"]:
                rows[:, b, :k] = _decode64(*got).permute(2, 0, 1, 3)
            elif st["opt"] is None:
                rows[b, :k] = got[0].double()
            else:
                rows.flatten(0, 1)[st["opt"][b, i // PAGE].long() * PAGE + i % PAGE] = got[0].double()
        return rows, wts, st["cnt"].view(-1)
    x = st["logits"].float().cpu().numpy()
    u = st["u"].cpu().numpy()
    s = [z.cpu().numpy() for z in st["set"]]
    if kind == "sample":
        if c["rows"] * c["V"] > 2.5e7:
            return None
        tok, pr = [], []
        for r in range(c["rows"]):
            w = _exact_kept(x[r], s[0][r], int(s[1][r]), s[2][r], s[3][r])
            tok.append(_exact_pick(w, u[r]))
            pr.append(w / max(w.sum(), 1e-300))
        tok = torch.tensor(tok, dtype=torch.int32, device=dev)
        return (tok, torch.from_numpy(np.stack(pr)).to(dev)) if c["probs"] else tok
    kept, tok = [], []
    ua, draft, nq = st["ua"].cpu().numpy(), st["draft"].cpu().numpy(), st["nq"].tolist()
    for b in range(c["B"]):
        for t in range(nq[b]):
            w = _exact_kept(x[b, t], s[0][b], int(s[1][b]), s[2][b], s[3][b])
            p = w / max(w.sum(), 1e-300)
            if t == nq[b] - 1:
                break
            d = draft[b, t]
            qrow = None if st["q"] is None else st["q"][b, t].double().cpu().numpy()
            if np.float64(ua[b, t]) * (1.0 if qrow is None else qrow[d]) < p[d]:
                continue
            if qrow is None:
                rest = p.copy()
                rest[d] = 0.0
            else:
                rest = np.maximum(p - qrow, 0.0)
            w = rest if rest.sum() > 0 else w
            break
        kept.append(t + 1)
        tok.append(_exact_pick(w, u[b]))
    return torch.tensor(kept, dtype=torch.int32, device=dev), torch.tensor(tok, dtype=torch.int32, device=dev)
