"""Drafted tokens with values that are not finite, at weights far below what 32 bits hold: a weight is above 0, however small it is."""
import math

import pytest
import torch

from paper_2311_02382_amd import lss
import _continuations as co
import _serving as sv

pytestmark = pytest.mark.gpu


def _hot(new, lengths, H, H_kv, d, page, dtype, seed, at):
    """Scores of about 1, but those of key `at` of sequence 0: 2^12 / sqrt(d), 360 to 512, so that all other weights are below 2^-500 of its own"""
    table, n_pages = sv.tables(lengths, page, seed)
    q = sv.normal(sum(new), H, d, seed=seed + 1, dtype=dtype)
    kc, vc = (sv.normal(n_pages, page, H_kv, d, seed=seed + i, dtype=dtype) for i in (2, 3))
    q[..., 0] = 64.0
    kc[..., 0] = 0.0
    kc[int(table[0, at // page]), at % page] = 0.0
    kc[int(table[0, at // page]), at % page, :, 0] = 64.0
    return q, kc, vc, table, sv.starts(new)


# (drafted, tokens, the key that outweighs all others, the drafted token whose values are not finite)
@pytest.mark.parametrize("dtype", sv.DTYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new,lengths,at,c", [
    ([3], [300], 10, 1),                                # another wavefront's
    ([4], [3000], 100, 1),                              # another part's
    ([70], [330], 20, 30), ([64], [5000], 200, 9),      # the same of many rows to a head of keys
    ([140] + [1] * 30, [400] + [9] * 30, 260 + 133, 5), ([140] + [1] * 30, [3000] + [9] * 30, 2860 + 133, 5),      # a later tile of the same wavefront's
])
def test_infinite_values_of_drafted_tokens_at_any_weight(dtype, d, new, lengths, at, c):
    H, H_kv, page = 4, 2, 16
    q, kc, vc, table, cu = _hot(new, lengths, H, H_kv, d, page, dtype, 40, at)
    n, first = new[0], lengths[0] - new[0]
    where = (int(table[0, (first + c) // page]), (first + c) % page)
    vc[where][:, 1], vc[where][:, 2], vc[where][:, 3] = math.inf, -math.inf, math.nan
    full = torch.full((n, 3), 0, dtype=torch.int64)
    full[:] = -1                                        # (every drafted token sees all of them)
    bits = torch.cat([full, torch.ones(sum(new) - n, 3, dtype=torch.int64)])
    for tree in (bits, None):
        out, lse = lss.lss_paged_attn_tree(q.cuda(), kc.cuda(), vc.cuda(), table.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda(), cu.cuda(),
                                           tree=None if tree is None else tree.cuda())
        torch.cuda.synchronize()
        want, want_lse, ob, lb = co.tree_attention(q, kc, vc, table, lengths, cu, tree)
        sees = torch.zeros(sum(new), dtype=torch.bool)
        sees[(0 if tree is not None else c):n] = True
        got = out[sees].float().cpu()
        assert bool((got[..., 1] == math.inf).all()) and bool((got[..., 2] == -math.inf).all()) and bool(got[..., 3].isnan().all())
        # (the oracle leaves values that are not finite out)
        sv.check(out[..., 4:], want[..., 4:], ob[..., 4:], "out")
        sv.check(out[~sees], want[~sees], ob[~sees], "rows that do not see it")
        sv.check(lse, want_lse, lb, "lse")
