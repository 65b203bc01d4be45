"""Beam search's choice where totals in 64 bits cannot tell a beam's logits apart: logits next to 0 beside a large log-sum-exp, scores that swallow them."""
import math

import pytest
import torch

from paper_2311_02382_amd import lss

pytestmark = pytest.mark.gpu


def _best(logits, scores, n_out):
    """[(k, v)] of a prompt, best first: by total in 64 bits, then by the lower beam, within a beam by the logits as they are, then by the lower token"""
    found = []
    for k in range(len(scores)):
        x = logits[k].double()
        lse = float(torch.logsumexp(x, 0))
        order = sorted(range(len(x)), key=lambda v: (-float(x[v]), v))[:n_out]
        found += [(-(float(scores[k]) + (float(x[v]) - lse)), k, -float(x[v]), v) for v in order]
    return [(k, v) for _, k, _, v in sorted(found)[:n_out]]


def _check(logits, scores, n_out):
    B, K = scores.shape
    _, parents, tokens, _ = lss.lss_beam_select(logits.cuda(), scores.cuda(), n_out)
    for b in range(B):
        want = _best(logits[b * K:(b + 1) * K], scores[b], n_out)
        got = [(int(p) - b * K, int(t)) for p, t in zip(parents[b], tokens[b])]
        assert got == want, (b, got, want)


# short rows and long ones, few chosen and many
FORMS = [(2, 1, 100, 1), (2, 1, 100, 3), (3, 2, 300, 8), (2, 4, 5000, 4), (2, 2, 5000, 40), (1, 20, 700, 64), (1, 32, 9000, 64)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("B,K,V,N", FORMS)
def test_logits_next_to_zero(dtype, B, K, V, N):
    # all 0 but a few that are as good as 0: below 0, above it, of any order of tokens; all beams alike, so that totals of different beams are equal too
    row = torch.zeros(V)
    gen = torch.Generator().manual_seed(V + N)
    some = torch.randperm(V, generator=gen)[:min(V // 2, 90)]
    row[some] = 2.0 ** (-60.0 - torch.arange(len(some)) % 37) * torch.where(torch.arange(len(some)) % 3 == 0, -1.0, 1.0)
    _check(row.to(dtype).expand(B * K, V).contiguous(), torch.full((B, K), -1.0), N)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("B,K,V,N", FORMS)
def test_scores_that_swallow_the_logits(dtype, B, K, V, N):
    logits = torch.randn(B * K, V, generator=torch.Generator().manual_seed(V + N)).to(dtype)
    scores = torch.full((B, K), -1e20)
    _check(logits, scores, N)
    scores[:, 0] = -5.0                                 # (one beam whose totals are told apart, in front of the others)
    _check(logits, scores, N)
    if K > 1:
        scores[:, 0], scores[:, -1] = -math.inf, -1e19
        assert int(lss.lss_beam_select(logits.cuda(), scores.cuda(), N)[1][0, 0]) == K - 1
