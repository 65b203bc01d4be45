"""Prompts, then tokens one by one, through append and both attentions: every step against its definition on the rows that the step before left."""
import pytest
import torch

from paper_2311_02382_amd import lss
import _serving as sv

pytestmark = pytest.mark.gpu


def _rotated(x, got, freq, interleaved, what):
    """Rows `got` of all tokens of a sequence are x, turned by their positions, rounded once"""
    want, slack = sv.rotate(x, torch.arange(len(x)), freq, interleaved)
    sv.check(got, want, slack + sv.HALF[x.dtype] * want.abs() * (0.0 if freq is None else 1.0), what)


def _attention(q, k, v):
    """out, lse and their bounds [tokens, H, ..] of a causal sequence"""
    G = q.shape[1] // k.shape[1]
    per_head = [sv.attention(q[:, h], k[:, h // G], v[:, h // G], torch.arange(len(q)) + 1, q.dtype) for h in range(q.shape[1])]
    return [torch.stack(x, 1) for x in zip(*per_head)]


def _off(got, want, bound):
    return float(((got - want).abs() > bound).double().mean())


@pytest.mark.parametrize("dtype", sv.DTYPES)
@pytest.mark.parametrize("H,H_kv,d,page,rot,interleaved", [(8, 2, 64, 16, 64, False), (4, 4, 128, 32, 64, True), (6, 1, 64, 64, 0, False), (4, 4, 64, 16, 32, False)])
def test_every_step_on_the_rows_that_are_kept(dtype, H, H_kv, d, page, rot, interleaved):
    prompts, steps = [33, 1, 140, 64, 600], 20
    total, B = [n + steps for n in prompts], len(prompts)
    table, n_pages = sv.tables(total, page, 300)
    q, k, v = ([sv.normal(n, h, d, seed=301 + 10 * b + i, dtype=dtype) for b, n in enumerate(total)] for i, h in ((1, H), (2, H_kv), (3, H_kv)))
    freq = sv.frequencies(rot) if rot else None
    k_cache, v_cache = (torch.full((n_pages, page, H_kv, d), float("nan"), dtype=dtype, device="cuda") for _ in range(2))
    lengths, cu, gpu_table = torch.tensor(prompts, dtype=torch.int32, device="cuda"), sv.starts(prompts).cuda(), table.cuda()
    options = dict(inv_freq=None if freq is None else freq.cuda(), interleaved=interleaved)
    first = [torch.cat([x[:n] for x, n in zip(xs, prompts)]).cuda() for xs in (q, k, v)]
    k_rot = torch.empty_like(first[1])
    q_rot, _ = lss.lss_paged_append(first[1], first[2], k_cache, v_cache, gpu_table, lengths, cu, q=first[0], k_rot=k_rot, **options)
    out, lse = lss.lss_packed_attn_fwd(q_rot, k_rot, first[2], cu)
    ranges = [slice(int(cu[b]), int(cu[b + 1])) for b in range(B)]
    q_kept, got, got_lse = ([[x[r]] for r in ranges] for x in (q_rot, out, lse.T))
    for i in range(steps):
        token = [torch.stack([x[n + i] for x, n in zip(xs, prompts)]).cuda() for xs in (q, k, v)]
        lengths += 1
        q_rot, _ = lss.lss_paged_append(token[1], token[2], k_cache, v_cache, gpu_table, lengths, q=token[0], **options)
        out, lse = lss.lss_paged_attn_decode(q_rot, k_cache, v_cache, gpu_table, lengths)
        for b in range(B):
            for kept, x in ((q_kept, q_rot), (got, out), (got_lse, lse)):
                kept[b].append(x[b:b + 1])
    k_cache, v_cache = k_cache.cpu(), v_cache.cpu()
    for b, n in enumerate(total):
        pages = table[b, :-(-n // page)].long()
        kb, vb = (x[pages].reshape(-1, H_kv, d)[:n] for x in (k_cache, v_cache))
        qb = torch.cat(q_kept[b]).cpu()
        _rotated(q[b], qb, freq, interleaved, f"queries of sequence {b}")
        _rotated(k[b], kb, freq, interleaved, f"keys of sequence {b}")
        assert torch.equal(vb, v[b]) and torch.equal(sv.bits(k_rot[ranges[b]]), sv.bits(kb[:prompts[b]]))
        want, want_lse, ob, lb = _attention(qb, kb, vb)
        sv.check(torch.cat(got[b]), want, ob, f"out of sequence {b}")
        sv.check(torch.cat(got_lse[b]), want_lse, lb, f"lse of sequence {b}")
        # what these bounds would not let pass: no results, rows that are not turned, a step that does not see its own token
        late = slice(prompts[b], n)
        assert _off(torch.zeros_like(want)[late], want[late], ob[late]) > 0.9
        if rot:
            plain = _attention(q[b], k[b], v[b])
            assert _off(plain[0][late], want[late], ob[late]) > 0.5 and _off(plain[1][late], want_lse[late], lb[late]) > 0.9
        G = H // H_kv
        score = (qb[late].double() * kb[late].double().repeat_interleave(G, 1)).sum(-1) / d ** 0.5         # of a token's own key
        rest = torch.log1p(-(score - want_lse[late]).exp()) + want_lse[late]
        assert _off(rest, want_lse[late], lb[late]) > 0.9
