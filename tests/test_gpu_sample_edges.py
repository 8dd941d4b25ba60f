"""Sampling where a row's weights lie about the cut of 2^-45, below which they count as zero: chunks of a row (8192 bf16
logits, 4096 in fp32) that hold nothing above it beside chunks that do."""
import numpy as np
import pytest
import torch

import paper_2606_24957_amd as D
from tests import sample_util as U

pytestmark = pytest.mark.gpu
DEV = "cuda"
LN2 = float(np.log(2.0))


def check(x, token, u, probs=None, settings=(1.0, 0, 1.0, 0.0)):
    w = U.kept_weights(x.double().cpu().numpy(), *settings)
    if u < 1.0:
        assert int(token) == U.pick(w, u), f"u {u}"
    else:
        assert w[int(token)] > 0, f"u {u}"
    if probs is not None:  # within 2^-45 of a weight, V of these in the sum, and one rounding
        ref = w / w.sum()
        tol = 2.0 ** -24 * ref + 2.0 ** -45 * (1 + ref * (1 + w.size))
        assert (np.abs(probs.double().cpu().numpy() - ref) <= tol * (1 + 1e-6)).all()


@pytest.mark.parametrize("V,best", [(16384, 12000), (16384, 100), (40001, 20000), (151936, 151935), (5000, 4999)])
@pytest.mark.parametrize("below", [31.0, 31.5, 32.0, 36.0, 39.0])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_no_filter_beside_chunks_below_the_cut(dtype, below, V, best):
    """A draw at either end of [0, 1] falls on a token that has a weight."""
    x = torch.full((4, V), -below, device=DEV)
    x[:, best] = 0.0
    x = x.to(dtype)
    u = torch.tensor([0.0, 2.0 ** -60, 1.0, 0.5], device=DEV)
    probs = torch.full((4, V), float("nan"), device=DEV)
    token, _ = D.sample(x, u, probs=probs)
    torch.cuda.synchronize()
    for b in range(4):
        check(x[b], token[b], float(u[b]), probs[b])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_verification_beside_chunks_below_the_cut(dtype):
    """The same rows after a rejected draft and after accepted ones."""
    V, best = 20000, 15000
    x = torch.full((2, 3, V), -32.0, device=DEV)
    x[:, :, best] = 0.0
    x = x.to(dtype)
    draft = torch.tensor([[best, best], [7, best]], dtype=torch.int32, device=DEV)
    ua, u = torch.full((2, 2), 0.5, device=DEV), torch.zeros(2, device=DEV)
    acc, token = D.verify_tokens(x, draft, ua, u)
    torch.cuda.synchronize()
    assert acc.tolist() == [3, 1] and token.tolist() == [best, best]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_only_token_of_a_chunk_just_above_the_cut(dtype):
    x = torch.full((2, 16384), float("-inf"), device=DEV)
    x[:, 12000] = 0.0
    x[0, 7] = x[1, 16000] = -31.0  # 2^-44.7
    x = x.to(dtype)
    u = torch.tensor([0.0, 1.0], device=DEV)
    token = D.sample(x, u)
    torch.cuda.synchronize()
    assert token.tolist() == [7, 16000]


def peaks(V, n, top, rest, place):
    """Every chunk of n tokens has one high logit (at its first, middle or last place), all others are `rest`."""
    x = torch.full((V,), float(rest))
    for c in range(0, V, n):
        size = min(n, V - c)
        x[c + {"first": 0, "middle": size // 2, "last": size - 1}[place]] = top - 0.0625 * (c // n)
    return x


@pytest.mark.parametrize("place", ["first", "middle", "last"])
@pytest.mark.parametrize("dtype,n", [(torch.float32, 4096), (torch.bfloat16, 8192)])
@pytest.mark.parametrize("V", [8190, 32000, 151936])
@pytest.mark.parametrize("top,rest,settings", [
    (0.0, -31.5, (1.0, 1000, 1.0, 0.0)),       # a top_k that the tokens with a weight do not reach
    (0.0, -31.5, (1.0, 3000, 0.999, 0.0)),
    (0.0, -31.5, (1.0, 1000, 1.0, 0.01)),
    (0.078125, -31.15, (1.0, 0, 1.0, 2.85e-14)),  # min_p ends in the eighth of an octave that the cut runs through
    (0.0, -31.75, (1.0, 512, 1.0, 0.0)),       # counts alone decide
    (0.0, -31.75, (1.0, 300, 0.9, 0.0)),
])
def test_lists_leave_out_what_has_no_weight(top, rest, settings, V, dtype, n, place):
    """Thousands of tokens just below the cut compete with none of those that have a weight for a place in a list."""
    x = peaks(V, n, top, rest, place)
    if V > 3 * n and settings[1] in (300, 512):  # a chunk whose best lies lower: its tokens below the cut are counted
        x[2 * n:3 * n] = float("-inf")
        x[2 * n:2 * n + 100] = rest
        x[2 * n + 50] = -0.25
    x = x.to(dtype).to(DEV).expand(4, V).contiguous()
    u = torch.tensor([0.0, 0.3, 0.7, 1.0 - 2.0 ** -24], device=DEV)
    probs = torch.full((4, V), float("nan"), device=DEV)
    kw = dict(temperature=settings[0], top_k=settings[1], top_p=settings[2], min_p=settings[3])
    token, _ = D.sample(x, u, probs=probs, **kw)
    torch.cuda.synchronize()
    for b in range(4):
        check(x[b], token[b], float(u[b]), probs[b], settings)
