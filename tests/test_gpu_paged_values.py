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
