"""Attention of packed sequences where keys or values are not finite: what the rows that see them get, and how long it takes."""
import math

import pytest
import torch

from paper_2311_02382_amd import lss
import _serving as sv
from test_gpu_packed_attn import _tensors, _want

pytestmark = pytest.mark.gpu

# every way through the kernels: groups of wavefronts in a workgroup, one group, keys that are split, more than 64 sequences
SHAPES = [([260, 30], [260, 30], 4, 2, 64), ([200], [1200], 4, 2, 128), ([64], [4100], 8, 2, 64), ([300], [3000], 2, 1, 128), ([17] * 70, [40] * 70, 4, 4, 64),
          ([1500], [1500], 32, 8, 64), ([1025], [1025], 16, 16, 128)]


def _inputs(n_q, n_k, H, H_kv, d, dtype, causal):
    """q, k, v, cu_q, cu_k on the GPU; the definition's results (CPU); tokens of every row's sequence that it sees [rows]"""
    q, k, v = (x.cuda() for x in _tensors(n_q, n_k, H, H_kv, d, dtype, 200))
    q *= 0.5
    cu_q, cu_k = sv.starts(n_q), sv.starts(n_k)
    want = [x.cpu() for x in _want(q, k, v, cu_q, cu_k, causal)]
    seen = torch.cat([(m - n + 1 + torch.arange(n)).clamp(0, m) if causal else torch.full((n,), m) for n, m in zip(n_q, n_k)])
    return q, k, v, cu_q.cuda(), cu_k.cuda(), want, seen


@pytest.mark.parametrize("dtype", sv.DTYPES)
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("n_q,n_k,H,H_kv,d", SHAPES)
def test_a_score_that_is_nan_is_one_in_both_results(dtype, causal, n_q, n_k, H, H_kv, d):
    # the first sequence's last rows see a key of NaN: out and lse of those are NaN, all others as they would be without it
    q, k, v, cu_q, cu_k, (want, want_lse, ob, lb), seen = _inputs(n_q, n_k, H, H_kv, d, dtype, causal)
    at = n_k[0] - n_q[0] // 2 - 1
    k[at] = float("nan")
    out, lse = lss.lss_packed_attn_fwd(q, k, v, cu_q, cu_k, causal=causal)
    hit = (torch.arange(len(seen)) < n_q[0]) & (seen > at)
    assert bool(hit.any()) and bool(torch.isnan(out[hit.cuda()]).all()) and bool(torch.isnan(lse[:, hit.cuda()]).all())
    sv.check(out[~hit.cuda()], want[~hit], ob[~hit], "out of the others")
    sv.check(lse[:, ~hit.cuda()], want_lse[:, ~hit], lb[:, ~hit], "lse of the others")


@pytest.mark.parametrize("dtype", sv.DTYPES)
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("n_q,n_k,H,H_kv,d", SHAPES)
def test_infinite_values_give_infinity(dtype, causal, n_q, n_k, H, H_kv, d):
    # column 1: +inf early, column 2: -inf in every seventh token, column 3: both signs, column 4: +inf in the last token, column 5: one NaN
    q, k, v, cu_q, cu_k, (want, want_lse, ob, lb), seen = _inputs(n_q, n_k, H, H_kv, d, dtype, causal)
    n = n_k[0]
    early, third = min(40, n // 2), n // 3
    v[early, :, 1], v[0:n:7, :, 2], v[0, :, 3], v[n - 1, :, 3] = math.inf, -math.inf, math.inf, -math.inf
    v[n - 1, :, 4], v[third, :, 5] = math.inf, math.nan
    out, lse = lss.lss_packed_attn_fwd(q, k, v, cu_q, cu_k, causal=causal)
    sv.check(lse, want_lse, lb, "lse")
    mine, out = torch.arange(len(seen)) < n_q[0], out.cpu()
    nan_at = lambda rows: torch.where(rows, math.nan, 0.0)
    expect = {1: torch.where(mine & (seen > early), math.inf, 0.0), 2: torch.where(mine & (seen > 0), -math.inf, 0.0),
              3: torch.where(mine & (seen >= n), math.nan, torch.where(mine & (seen > 0), math.inf, 0.0)),
              4: torch.where(mine & (seen >= n), math.inf, 0.0), 5: nan_at(mine & (seen > third))}
    for column in range(d):
        special = expect.get(column, torch.zeros(len(seen)))
        free = special == 0
        sv.check(out[free][..., column], want[free][..., column], ob[free][..., column], f"column {column}")
        got, value = out[~free][..., column].float(), special[~free][:, None].expand(-1, H)
        assert torch.equal(torch.isnan(got), torch.isnan(value)) and bool(((got == value) | torch.isnan(value)).all()), column


@pytest.mark.parametrize("dtype", sv.DTYPES)
def test_values_that_are_not_finite_cost_bounded_time(dtype):
    # 4096 rows of 8 heads of 64, 2 of keys: a row that is done over walks 2048 keys on average; 64 at a time in about 3000 cycles that is 0.1 ms and 32 rows of a
    # wavefront 3 ms at most, beside 0.05 to 0.2 ms of the call.  A NaN among the scores does over nothing.
    q, k, v = (x.cuda() for x in _tensors([4096], [4096], 8, 2, 64, dtype, 210))
    cu = sv.starts([4096]).cuda()

    def least():
        times = []
        for _ in range(5):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            lss.lss_packed_attn_fwd(q, k, v, cu)
            b.record()
            b.synchronize()
            times.append(a.elapsed_time(b))
        return min(times)

    least()
    clean = least()
    v[40, 0, 7] = math.inf
    values = least()
    v[40, 0, 7], k[0] = 1.0, math.nan
    keys = least()
    print(f"clean {clean * 1e3:.0f} us, a value of infinity {values * 1e3:.0f}, a key of NaN {keys * 1e3:.0f}")
    assert values < clean + 4.0 and keys < 3 * clean + 0.05
