"""Sampling and the verification of drafted tokens on the GPU against their definition in float64: tokens and accepted
counts equal, probabilities to the rounding of fp32."""
import numpy as np
import pytest
import torch

import paper_2606_24957_amd as D
from tests import sample_util as U

pytestmark = pytest.mark.gpu
DEV = "cuda"
F = torch.float32


def rows(kind, B, V, seed):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((B, V)) * 2
    if kind == "peaked":
        for b in range(B):
            at = rng.choice(V, min(V, 20), replace=False)
            x[b, at] += rng.uniform(5, 14, at.size)
    elif kind == "flat":
        x *= 0.01
    elif kind == "equal":
        x[:] = 1.5
    elif kind == "few":
        x[:] = rng.choice([0.0, 1.0, 1.5], (B, V))
    elif kind == "masked":
        x[rng.random((B, V)) < 0.9] = -np.inf
        x[:, :: 7] = float(torch.finfo(torch.float32).min)
        x[0] = -np.inf
        x[-1] = float(torch.finfo(torch.float32).min)
        if B > 2:
            x[1, : V // 2] = np.nan
            x[2] = np.nan
        if B > 3:
            x[3, V // 3] = np.inf
            x[3, V // 2] = np.inf
    elif kind == "wide":
        x *= 30
    elif kind == "huge":
        x *= 1e37
    return x


def check(x, u, settings, probs=None, token=None):
    """settings: per-row lists of temperature, top_k, top_p, min_p; x as the kernel saw it (float64)."""
    for b in range(x.shape[0]):
        w = U.kept_weights(x[b], *(s[b] for s in settings))
        assert int(token[b]) == U.pick(w, u[b]), f"row {b} of settings {[s[b] for s in settings]}"
        if probs is not None:
            ref = w / w.sum() if w.sum() > 0 else w
            # a weight and a sum are within 2^-45 of the largest of theirs (a sum: of V times that), then one rounding
            tol = 2.0 ** -24 * ref + 2.0 ** -45 * (1 + ref) + 2.0 ** -45 * ref * x.shape[1]
            assert (np.abs(probs[b] - ref) <= tol * (1 + 1e-6)).all(), f"row {b}"


SETTINGS = [  # temperature, top_k, top_p, min_p
    (1.0, 0, 1.0, 0.0), (0.7, 20, 0.9, 0.0), (1.3, 0, 0.95, 0.0), (0.0, 5, 0.5, 0.1), (1.0, 0, 1.0, 0.05),
    (0.8, 1, 1.0, 0.0), (1.0, 50, 1.0, 0.02), (2.0, 0, 0.5, 0.3), (1.0, 3000, 0.99, 0.0), (0.05, 0, 0.999, 0.0),
    (1.0, 0, 0.0, 0.0), (1.5, 2000, 1.0, 0.0), (100.0, 0, 0.7, 0.0), (1.0, 7, 0.3, 1.0), (1.0, 10 ** 9, 2.0, -1.0),
]


@pytest.mark.parametrize("kind", ["normal", "peaked", "flat", "equal", "few", "masked", "wide", "huge"])
@pytest.mark.parametrize("V,dtype", [(1, F), (2, torch.bfloat16), (63, F), (1000, torch.bfloat16), (4097, F),
                                     (32000, torch.bfloat16), (50257, F)])
def test_sample(V, dtype, kind):
    B = len(SETTINGS)
    x = torch.from_numpy(rows(kind, B, V, V)).to(torch.float32).to(dtype).to(DEV)
    u = torch.rand(B, generator=torch.Generator().manual_seed(V)).to(DEV)
    u[0], u[1] = 0.0, 1.0 - 2.0 ** -24
    cols = list(zip(*SETTINGS))
    kw = dict(temperature=torch.tensor(cols[0], device=DEV), top_k=torch.tensor(cols[1], dtype=torch.int32, device=DEV),
              top_p=torch.tensor(cols[2], device=DEV), min_p=torch.tensor(cols[3], device=DEV))
    probs = torch.full((B, V), float("nan"), device=DEV)
    token, _ = D.sample(x, u, probs=probs, **kw)
    torch.cuda.synchronize()
    check(x.double().cpu().numpy(), u.cpu().numpy(), cols, probs.double().cpu().numpy(), token)
    again = D.sample(x, u, **kw)
    assert torch.equal(again, token)


@pytest.mark.parametrize("setting", SETTINGS)
@pytest.mark.parametrize("V,kind", [(262144, "normal"), (151936, "peaked"), (151937, "few")])
def test_large_vocabularies(V, kind, setting):
    x = torch.from_numpy(rows(kind, 3, V, 7)).to(torch.float32).to(DEV)
    for dtype in (F, torch.bfloat16):
        y = x.to(dtype)
        u = torch.tensor([0.1, 0.5, 0.999], device=DEV)
        token = D.sample(y, u, temperature=setting[0], top_k=setting[1], top_p=setting[2], min_p=setting[3])
        torch.cuda.synchronize()
        check(y.double().cpu().numpy(), u.cpu().numpy(), [[s] * 3 for s in setting], token=token)


def test_top_p_ends_inside_equal_logits():
    """Of equal logits those with the lowest indexes stay."""
    x = torch.full((4, 1000), -5.0, dtype=torch.bfloat16, device=DEV)
    x[:, 100:900:2] = 3.0
    u = torch.tensor([0.0, 0.4999, 0.9999, 0.75], device=DEV)
    probs = torch.empty((4, 1000), device=DEV)
    token, _ = D.sample(x, u, top_p=0.5, probs=probs)
    p = 400 + 600 * np.exp(-8.0)
    n = int(np.ceil(0.5 * p))  # kept
    assert token.tolist() == [100, 100 + 2 * int(0.4999 * n), 100 + 2 * (n - 1), 100 + 2 * int(0.75 * n)]
    assert ((probs > 0).sum(1) == n).all() and (probs[0, 100:100 + 2 * n:2] > 0).all()


def test_strided_rows_and_streams():
    V = 1003
    base = torch.randn((6, 3 * V + 1), device=DEV)
    u = torch.rand(6, device=DEV)
    for dtype in (F, torch.bfloat16):
        for off in (0, 1, 5):
            x = base.to(dtype)[:, off:off + V]
            want = D.sample(x.contiguous(), u, top_k=30, top_p=0.9)
            assert torch.equal(D.sample(x, u, top_k=30, top_p=0.9), want)
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                got = D.sample(x, u, top_k=30, top_p=0.9)
            side.synchronize()
            assert torch.equal(got, want)


def window(B, T, V, seed, drawn, dtype):
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = (2 * torch.randn((B, T, V), generator=g, device=DEV)).to(dtype)
    near = x[:, :T - 1].float() + 0.5 * torch.randn((B, T - 1, V), generator=g, device=DEV)
    q = None
    if drawn:
        q = torch.softmax(near * 1.5, -1)
        draft = torch.multinomial(q.reshape(-1, V), 1, generator=g).view(B, T - 1).to(torch.int32) if T > 1 else \
            torch.zeros((B, 0), dtype=torch.int32, device=DEV)
    else:
        draft = near.argmax(-1).to(torch.int32)
    return x, draft, torch.rand((B, T - 1), generator=g, device=DEV), torch.rand(B, generator=g, device=DEV), q


def check_window(x, draft, ua, u, q, nq, settings, got):
    acc, tok = (z.tolist() for z in got)
    xs = x.double().cpu().numpy()
    for b in range(x.shape[0]):
        s = [z[b] if isinstance(z, (list, tuple)) else z for z in settings]
        want = U.verify(xs[b, :nq[b]], draft[b].tolist(), ua[b].cpu().numpy(), float(u[b]), s,
                        None if q is None else q[b].cpu().numpy())
        assert (acc[b], tok[b]) == want, f"sequence {b}"


@pytest.mark.parametrize("drawn", [False, True])
@pytest.mark.parametrize("B,T,V,dtype", [(1, 1, 100, F), (3, 2, 33, torch.bfloat16), (16, 5, 1000, F),
                                         (7, 9, 5003, torch.bfloat16), (2, 64, 257, F), (4, 4, 40000, torch.bfloat16)])
def test_verify(B, T, V, dtype, drawn):
    x, draft, ua, u, q = window(B, T, V, V + T, drawn, dtype)
    nq = [max(0, T - b % 3) for b in range(B)]
    settings = ([SETTINGS[b % 8][0] for b in range(B)], [SETTINGS[b % 8][1] for b in range(B)],
                [SETTINGS[b % 8][2] for b in range(B)], [SETTINGS[b % 8][3] for b in range(B)])
    kw = dict(temperature=torch.tensor(settings[0], device=DEV), top_p=torch.tensor(settings[2], device=DEV),
              top_k=torch.tensor(settings[1], dtype=torch.int32, device=DEV), min_p=torch.tensor(settings[3], device=DEV))
    got = D.verify_tokens(x, draft, ua, u, draft_probs=q, n_query=torch.tensor(nq, dtype=torch.int32, device=DEV), **kw)
    torch.cuda.synchronize()
    check_window(x, draft, ua, u, q, nq, settings, got)


def test_verify_at_the_edges():
    """Drafts outside the vocabulary, certain and impossible ones, empty windows, a row that masks everything."""
    B, T, V = 8, 4, 500
    x, draft, ua, u, q = window(B, T, V, 5, True, F)
    draft[0] = torch.tensor([-1, 3, 4])
    draft[1, 1] = V
    x[2, :3] = -50.0
    for t in range(3):
        x[2, t, draft[2, t]] = 50.0     # accepted
    x[3, 0, draft[3, 0]] = -float("inf")  # impossible
    x[4, 2] = -float("inf")
    x[5] = -float("inf")
    q[6, :, :] = 0.0                      # drawn from nothing: accepted where the target has any weight
    nq = [4, 4, 4, 4, 4, 4, 4, 0]
    got = D.verify_tokens(x, draft, ua, u, draft_probs=q, n_query=torch.tensor(nq, dtype=torch.int32, device=DEV))
    torch.cuda.synchronize()
    check_window(x, draft, ua, u, q, nq, (1.0, 0, 1.0, 0.0), got)
    assert int(got[0][2]) == 4 and int(got[0][3]) == 1 and int(got[0][6]) == 4 and got[1][5] == -1


def test_verify_draws_what_the_target_would():
    """Drafts from another distribution, accepted and replaced: the first token is distributed as the target's."""
    V, B = 8, 40000
    g = torch.Generator(device=DEV).manual_seed(1)
    lt, ld = torch.randn(V, generator=g, device=DEV), torch.randn(V, generator=g, device=DEV)
    p, q = torch.softmax(lt, -1), torch.softmax(ld, -1)
    draft = torch.multinomial(q, B, replacement=True, generator=g).to(torch.int32).view(B, 1)
    ua, u = (torch.rand((B, 1), generator=g, device=DEV) for _ in range(2))
    acc, tok = D.verify_tokens(lt.expand(B, 2, V).contiguous()[:32000], draft[:32000], ua[:32000], u[:32000, 0].contiguous(),
                               draft_probs=q.expand(B, 1, V)[:32000])
    first = torch.where(acc == 2, draft[:32000, 0], tok).cpu()
    freq = torch.bincount(first, minlength=V).double() / 32000
    # six standard deviations of a frequency
    assert ((freq - p.double().cpu()).abs() < 6 * (p.double().cpu() / 32000).sqrt()).all()


def test_captured_and_replayed():
    B, T, V = 5, 4, 9001
    x, draft, ua, u, q = window(B, T, V, 11, True, torch.bfloat16)
    nq = [4, 4, 3, 2, 1]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        v = D.plan_verify_tokens(x, draft, ua, u, draft_probs=q, top_p=0.9, n_query=torch.tensor(nq, dtype=torch.int32, device=DEV))
        s = D.plan_sample(x[:, 0], u, top_k=40)
        v(), s()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        v(), s()
    for seed in (21, 22, 23):
        y = window(B, T, V, seed, True, torch.bfloat16)
        for old, new in zip((x, draft, ua, u, q), y):
            old.copy_(new)
        D.sample(torch.randn((3, 777), device=DEV), torch.rand(3, device=DEV), top_p=0.5)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        check_window(x, draft, ua, u, q, nq, (1.0, 0, 0.9, 0.0), v.result)
        check(x[:, 0].double().cpu().numpy(), u.cpu().numpy(), ([1.0] * B, [40] * B, [1.0] * B, [0.0] * B), token=s.result)


@pytest.mark.parametrize("kind", ["normal", "peaked", "few"])
@pytest.mark.parametrize("V,dtype", [(5003, F), (40000, torch.bfloat16)])
def test_all_filters_together(V, dtype, kind):
    """Every filter with every other: what min_p leaves out still belongs to the sum that top_p is a part of."""
    cols = list(zip(*[(t, k, p, m) for t in (1.0, 0.6) for k in (0, 20, 400, 700, 3000) for p in (1.0, 0.95, 0.6)
                      for m in (0.0, 0.001, 0.05, 0.5)]))
    B = len(cols[0])
    x = torch.from_numpy(rows(kind, B, V, V + 1)).to(torch.float32).to(dtype).to(DEV)
    u = torch.rand(B, generator=torch.Generator().manual_seed(V)).to(DEV)
    kw = dict(temperature=torch.tensor(cols[0], device=DEV), top_k=torch.tensor(cols[1], dtype=torch.int32, device=DEV),
              top_p=torch.tensor(cols[2], device=DEV), min_p=torch.tensor(cols[3], device=DEV))
    probs = torch.full((B, V), float("nan"), device=DEV)
    token, _ = D.sample(x, u, probs=probs, **kw)
    torch.cuda.synchronize()
    check(x.double().cpu().numpy(), u.cpu().numpy(), cols, probs.double().cpu().numpy(), token)


@pytest.mark.parametrize("V,dtype", [(300, F), (9001, F), (32000, torch.bfloat16)])
def test_small_weights_stay_where_nothing_ends_the_set(V, dtype):
    """A top_k beyond the tokens that have a weight keeps them all, down to 2^-45 of the largest."""
    x = np.full((6, V), -1e30)
    at = np.random.default_rng(V).permutation(V)[:120]
    x[:, at] = -np.arange(120) * 0.25  # weights to e^-29.75 = 2^-42.9
    x[3:, at] *= 1.04                  # to 2^-44.6
    x = torch.from_numpy(x).to(torch.float32).to(dtype).to(DEV)
    u = torch.tensor([0.0, 0.5, 1.0 - 2.0 ** -24] * 2, device=DEV)
    cols = ([1.0] * 6, [V - 1] * 6, [1.0] * 6, [0.0] * 6)
    probs = torch.full((6, V), float("nan"), device=DEV)
    token, _ = D.sample(x, u, top_k=V - 1, probs=probs)
    torch.cuda.synchronize()
    check(x.double().cpu().numpy(), u.cpu().numpy(), cols, probs.double().cpu().numpy(), token)
