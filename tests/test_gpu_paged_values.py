"""Attention of one token per sequence over a paged cache: values that are infinite, and how exactly a weight enters."""
import math

import pytest
import torch

from paper_2311_02382_amd import lss
import _serving as sv
from test_gpu_paged_decode import _inputs, _want

CASES = [([3, 1, 40, 512], 4, 2, 64, 16), ([700, 33, 2500], 8, 2, 64, 32), ([1300, 90], 4, 4, 128, 16), ([600, 17], 20, 1, 64, 16), ([2000, 130], 33, 1, 128, 64)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", sv.DTYPES)
@pytest.mark.parametrize("lengths,H,H_kv,d,page", CASES)
def test_infinite_values_give_infinity(dtype, lengths, H, H_kv, d, page):
    # column 1: one +inf, column 2: several -inf, column 3: both, column 4: +inf in the last token, column 5: one NaN; every weight is above 0
    q, kc, vc, table = _inputs(lengths, H, H_kv, d, page, dtype, 40)
    q *= 0.5
    put = vc.clone()

    def at(b, p):
        return int(table[b, p // page]), p % page

    sign = {1: math.inf, 2: -math.inf, 3: math.nan, 4: math.inf, 5: math.nan}
    for b, n in enumerate(lengths):
        put[(*at(b, n // 2), slice(None), 1)] = math.inf
        for p in range(0, n, 7):
            put[(*at(b, p), slice(None), 2)] = -math.inf
        put[(*at(b, 0), slice(None), 3)] = math.inf
        put[(*at(b, n - 1), slice(None), 4)] = math.inf
        put[(*at(b, n // 3), slice(None), 5)] = math.nan
        if n > 1:
            put[(*at(b, n - 1), slice(None), 3)] = -math.inf
    out, lse = lss.lss_paged_attn_decode(*(x.cuda() for x in (q, kc, put, table, torch.tensor(lengths, dtype=torch.int32))))
    want, want_lse, ob, lb = _want(q, kc, vc, table, lengths)
    sv.check(lse, want_lse, lb, "lse")
    out = out.double().cpu()
    for b, n in enumerate(lengths):
        for column, value in sign.items():
            if column == 3 and n == 1:
                value = math.inf
            got = out[b, :, column]
            assert bool((torch.isnan(got) if math.isnan(value) else got == value).all()), (b, column, got)
    clean = [c for c in range(d) if c not in sign]
    sv.check(out[..., clean], want[..., clean], ob[..., clean], "out of the other columns")


def _cancelling(lengths, H, d, page):
    """bf16 inputs of a head of keys per query head: two tokens of a sequence outweigh all others by e^11 or so, and their weighted values cancel but for the
    rounding of the second one.  So a weight's error shows, where a result of the values' own size would hide it behind its own rounding."""
    q, kc, vc, table = _inputs(lengths, H, H, d, page, torch.bfloat16, 60)
    flat_k, flat_v = kc.view(-1, H, d), vc.view(-1, H, d)
    for b, n in enumerate(lengths):
        rows = torch.tensor([int(table[b, p // page]) * page + p % page for p in range(n)])
        one, two = rows[n // 7], rows[n - 1]
        near = sv.normal(2, H, d, seed=70 + b)
        flat_k[rows] = (-1.5 * q[b].float() * 8 / d ** 0.5).to(torch.bfloat16)
        flat_k[one], flat_k[two] = near[0], near[1]
        w = ((flat_k[torch.stack([one, two])].double() * q[b].double()).sum(-1) / d ** 0.5).exp()
        flat_v[two] = (-(w[0] / w[1])[:, None] * flat_v[one].double()).to(torch.bfloat16)
    return q, kc, vc, table


def _two_parts_bound(q, kc, vc, table, lengths):
    """(out, bound of its error, scores, values) per sequence: the result rounded once, and weights off by 2^-16 and by what _serving.attention allows for exponential, scores and sums"""
    H, d = q.shape[1:]
    page = kc.shape[1]
    for b, n in enumerate(lengths):
        rows = torch.tensor([int(table[b, p // page]) * page + p % page for p in range(n)])
        k, v = kc.view(-1, H, d)[rows].double(), vc.view(-1, H, d)[rows].double()
        x = q[b].double()
        score = (k * x).sum(-1) / d ** 0.5                                          # [n, H]
        size = ((k.abs() * x.abs()).sum(-1) / d ** 0.5).amax(0)
        weight = score.softmax(0)
        out, absolute = torch.einsum("nh,nhd->hd", weight, v), torch.einsum("nh,nhd->hd", weight, v.abs())
        each = (d + 2) * 2.0 ** -24 * size + 2.0 ** -21 + (n + 8) * 2.0 ** -24
        yield out, sv.HALF[torch.bfloat16] * out.abs() + (2.0 ** -16 + 2 * each)[:, None] * absolute, score, v


LENGTHS = [2, 3, 17, 64, 512, 700, 1900]


@pytest.mark.parametrize("d", [64, 128])
def test_the_bound_tells_two_parts_of_a_weight_from_one(d):
    # on the CPU: weights rounded to bf16 break it for half of all results at least, weights of two parts never
    inputs = _cancelling(LENGTHS, 4, d, 16)
    for out, bound, score, v in _two_parts_bound(*inputs, LENGTHS):
        p = (score - score.amax(0)).exp().float()
        cut = (p.view(torch.int32) & -65536).view(torch.float32)
        for parts, broken in ((p.to(torch.bfloat16).double(), True), (cut.double() + (p - cut).to(torch.bfloat16).double(), False)):
            got = torch.einsum("nh,nhd->hd", parts, v) / p.double().sum(0)[:, None]
            off = ((got.to(torch.bfloat16).double() - out).abs() > bound).double().mean()
            assert off > 0.5 if broken else off == 0, (len(score), float(off))


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lengths", [LENGTHS, LENGTHS[:5]])
def test_weights_are_not_rounded_to_bf16(lengths, d):
    q, kc, vc, table = _cancelling(lengths, 4, d, 16)
    out, _ = lss.lss_paged_attn_decode(*(x.cuda() for x in (q, kc, vc, table, torch.tensor(lengths, dtype=torch.int32))))
    for b, (want, bound, _, _) in enumerate(_two_parts_bound(q, kc, vc, table, lengths)):
        sv.check(out[b], want, bound, f"sequence of {lengths[b]}")
