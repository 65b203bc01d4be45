"""Attention of drafted tokens over a paged cache, against its definition in 64 bits."""
import math

import pytest
import torch

from paper_2311_02382_amd import lss
import _continuations as co
import _serving as sv

pytestmark = pytest.mark.gpu


def _inputs(new, lengths, H, H_kv, d, page, dtype, seed, words=1, extra=0, more_rows=0):
    table, n_pages = sv.tables(lengths, page, seed, extra=extra)
    gen = torch.Generator().manual_seed(seed)
    rows = sum(new) + more_rows
    q = sv.normal(rows, H, d, seed=seed + 1, dtype=dtype)
    kc, vc = (sv.normal(n_pages, page, H_kv, d, seed=seed + i, dtype=dtype) for i in (2, 3))
    tree = torch.cat([co.random_tree(n, words, gen) for n in new] + [torch.zeros(more_rows, words, dtype=torch.int64)])
    return q, kc, vc, table, sv.starts(new), tree


def _run(new, lengths, H, H_kv, d, page, dtype=torch.bfloat16, seed=1, words=1, max_len=None, inputs=None, tree=True, **more):
    q, kc, vc, table, cu, bits = inputs or _inputs(new, lengths, H, H_kv, d, page, dtype, seed, words, **more)
    bits = bits if tree else None
    out, lse = torch.full(q.shape, 7.0, dtype=dtype, device="cuda"), torch.full(q.shape[:2], 7.0, device="cuda")
    lss.lss_paged_attn_tree(q.cuda(), kc.cuda(), vc.cuda(), table.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda(), cu.cuda(), tree=None if bits is None else bits.cuda(),
                            max_len=max_len, out=out, lse=lse)
    torch.cuda.synchronize()
    want, want_lse, ob, lb = co.tree_attention(q, kc, vc, table, lengths, cu, bits, max_len)
    # rows of no sequence are left as they were
    for x, bound in ((want, ob), (want_lse, lb)):
        bound[x.isnan()] = 0.0
        x[x.isnan()] = 7.0
    sv.check(out, want, ob, "out")
    sv.check(lse, want_lse, lb, "lse")
    return out, lse


@pytest.mark.parametrize("dtype", sv.DTYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("tree", [True, False])
def test_lengths_around_every_tile(dtype, d, page, tree):
    lengths = [1, 2, 15, 16, 17, 31, 32, 33, 47, 63, 64, 65, 100, 127, 128, 129, 191, 255, 256, 257, 0]
    new = [1, 1, 5, 16, 1, 7, 32, 3, 40, 63, 64, 2, 9, 1, 33, 17, 64, 1, 10, 20, 0]
    _run(new, lengths, 4, 2, d, page, dtype, seed=100, tree=tree)


@pytest.mark.parametrize("dtype", sv.DTYPES)
@pytest.mark.parametrize("H,H_kv", [(1, 1), (3, 3), (2, 1), (6, 2), (7, 1), (16, 1), (17, 1), (32, 2), (33, 1), (40, 2), (64, 1)])
def test_groups_of_heads(dtype, H, H_kv):
    _run([5, 21], [77, 300], H, H_kv, 64, 16, dtype, seed=200 + H)
    _run([9], [130], H, H_kv, 128, 32, dtype, seed=300 + H)


@pytest.mark.parametrize("dtype", sv.DTYPES)
@pytest.mark.parametrize("new,lengths,H,H_kv,d,page", [([13], [3000], 8, 2, 128, 64), ([5, 1, 30], [2097, 1, 700], 4, 4, 64, 16), ([64], [4001], 4, 1, 64, 256),
                                                       ([3] * 4, [1500] * 4, 16, 2, 128, 1024), ([1, 0, 33, 20], [1500, 0, 33, 1999], 5, 5, 128, 128)])
def test_long_sequences(dtype, new, lengths, H, H_kv, d, page):
    for tree in (True, False):
        _run(new, lengths, H, H_kv, d, page, dtype, seed=400, tree=tree)


@pytest.mark.parametrize("dtype", sv.DTYPES)
def test_many_drafted_tokens(dtype):
    # trees of several words; chains far longer than a tile of rows
    _run([64, 65, 130, 1], [64, 400, 150, 1], 4, 2, 64, 16, dtype, seed=500, words=3)
    _run([300, 7], [900, 500], 6, 2, 64, 32, dtype, seed=501, tree=False)
    _run([200], [200], 2, 2, 128, 16, dtype, seed=502, words=4)


def test_a_chunk_of_a_long_prompt():
    _run([700], [2700], 8, 2, 128, 64, seed=510, tree=False)
    _run([513, 100], [1800, 100], 4, 4, 64, 16, seed=511, tree=False)


def test_more_parts_than_two_a_compute_unit():
    # 192 tiles of rows of 90 to 94 rounds: four parts each where three workgroups are resident, two where two are
    for tree in (True, False):
        _run([64] * 24, [6000 - 11 * b for b in range(24)], 16, 4, 64, 32, seed=515, tree=tree)


def test_many_sequences():
    _run([b % 4 for b in range(200)], [(37 * b) % 90 + 3 for b in range(200)], 8, 2, 64, 16, seed=520)
    _run([1 + b % 3 for b in range(90)], [(67 * b) % 900 + 3 for b in range(90)], 4, 1, 128, 32, seed=521)


@pytest.mark.parametrize("dtype", sv.DTYPES)
@pytest.mark.parametrize("d", [64, 128])
def test_masks_of_every_kind(dtype, d):
    # nothing at all: only the tokens in front; everything; a row that sees what comes after it; words that are too few; the sign bit
    new, lengths = [70, 3, 5, 64, 2], [70, 3, 40, 90, 700]
    inputs = list(_inputs(new, lengths, 4, 2, d, 16, dtype, 600))
    gen = torch.Generator().manual_seed(601)
    bits = torch.randint(-2 ** 63, 2 ** 63 - 1, (sum(new), 1), generator=gen)
    bits[0], bits[1], bits[70:73], bits[73], bits[74] = 0, -1, 0, 0, -1
    bits[80] = -2 ** 63
    inputs[5] = bits
    out, lse = _run(new, lengths, 4, 2, d, 16, dtype, inputs=inputs)
    assert bool((lse[0] == -math.inf).all()) and bool((out[70:73] == 0).all())          # rows that see nothing


@pytest.mark.parametrize("dtype", sv.DTYPES)
@pytest.mark.parametrize("tree", [True, False])
def test_lengths_shorter_than_what_is_drafted(dtype, tree):
    # fewer tokens than rows: the last of them are the keys; lengths below 0 and past the tables; a bound on the lengths
    _run([20, 8, 5, 4], [7, 0, -5, 5], 4, 2, 64, 16, dtype, seed=610, tree=tree)
    _run([4, 6], [2 ** 31 - 1, 40], 4, 2, 64, 16, dtype, tree=tree, inputs=_inputs([4, 6], [48, 40], 4, 2, 64, 16, dtype, 611))
    _run([4, 6, 9], [40, 200, 513], 4, 2, 64, 16, dtype, seed=612, max_len=200, tree=tree)
    _run([4, 6], [40, 200], 4, 2, 64, 16, dtype, seed=613, max_len=0, tree=tree)


@pytest.mark.parametrize("dtype", sv.DTYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("garbage", [math.nan, math.inf, -3e38])
@pytest.mark.parametrize("tree", [True, False])
def test_what_a_row_does_not_see_stays_there(dtype, d, garbage, tree):
    # the same rows with the values and keys of a drafted token spoilt: rows that do not see it keep their bits, those that do are spoilt as the definition has it;
    # and what lies behind the last token
    new, lengths = [7, 12, 1, 40], [7, 33, 16, 500]
    q, kc, vc, table, cu, bits = _inputs(new, lengths, 6, 2, d, 16, dtype, 700, extra=2)
    clean = [x.cuda() for x in (q, kc, vc, table, torch.tensor(lengths, dtype=torch.int32), cu)]
    kw = dict(tree=bits.cuda() if tree else None)
    want, want_lse = lss.lss_paged_attn_tree(*clean, **kw)
    exact, exact_lse, ob, lb = co.tree_attention(q, kc, vc, table, lengths, cu, bits if tree else None)
    mine = torch.zeros(kc.shape[:2], dtype=torch.bool)
    for b, n in enumerate(lengths):
        for p in range(n):
            mine[int(table[b, p // 16]), p % 16] = True
    for what in ("v", "k"):
        bad_k, bad_v = kc.clone(), vc.clone()
        bad_k[~mine], bad_v[~mine] = garbage, garbage
        sees = torch.zeros(len(q), dtype=torch.bool)
        for b, n in enumerate(new):
            c = n // 2
            p = lengths[b] - n + c
            (bad_v if what == "v" else bad_k)[int(table[b, p // 16]), p % 16] = garbage
            for i in range(n):
                sees[int(cu[b]) + i] = (int(bits[int(cu[b]) + i, 0]) >> c & 1) != 0 if tree else c <= i
        out, lse = lss.lss_paged_attn_tree(clean[0], bad_k.cuda(), bad_v.cuda(), *clean[3:], **kw)
        torch.cuda.synchronize()
        # (a key that other rows see may make them raise their running maximum, and with them the rows beside them: other roundings, within the bounds)
        sv.check(out[~sees], exact[~sees], ob[~sees], "out"), sv.check(lse[~sees], exact_lse[~sees], lb[~sees], "lse")
        if what == "v":
            assert torch.equal(sv.bits(out[~sees]), sv.bits(want[~sees])) and torch.equal(sv.bits(lse), sv.bits(want_lse))
            spoilt = out[sees].float().cpu()
            if math.isnan(garbage):
                assert bool(spoilt.isnan().all())
            elif math.isinf(garbage):
                assert bool((spoilt == math.inf).all())


@pytest.mark.parametrize("dtype", sv.DTYPES)
def test_infinite_values_in_front_of_the_drafted_tokens(dtype):
    new, lengths = [5, 40], [40, 700]
    q, kc, vc, table, cu, bits = _inputs(new, lengths, 4, 2, 64, 16, dtype, 720)
    q *= 0.5
    for b in range(2):
        vc[int(table[b, 0]), 3, :, 1], vc[int(table[b, 1]), 0, :, 2] = math.inf, -math.inf
        vc[int(table[b, 0]), 5, :, 3], vc[int(table[b, 1]), 2, :, 3] = math.inf, -math.inf
    for tree in (bits.cuda(), None):
        out, lse = lss.lss_paged_attn_tree(q.cuda(), kc.cuda(), vc.cuda(), table.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda(), cu.cuda(), tree=tree)
        assert bool((out[..., 1] == math.inf).all()) and bool((out[..., 2] == -math.inf).all()) and bool(out[..., 3].isnan().all())
        want, want_lse, ob, lb = co.tree_attention(q, kc, vc, table, lengths, cu, None if tree is None else bits)
        sv.check(out[..., 4:], want[..., 4:], ob[..., 4:], "out")
        sv.check(lse, want_lse, lb, "lse")


@pytest.mark.parametrize("dtype", sv.DTYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("tree", [True, False])
def test_numbers_that_are_no_page(dtype, d, tree):
    new, lengths = [10, 64, 3, 33, 40], [40, 64, 100, 33, 700]
    q, kc, vc, table, cu, bits = _inputs(new, lengths, 4, 2, d, 16, dtype, 800)
    n_pages = len(kc)
    kc[-1], vc[-1] = math.nan, math.nan
    kc[0], vc[0] = math.nan, math.nan
    table[table == 0] = -1
    table[table == n_pages - 1] = n_pages
    table[0, 1], table[1, :] = -1, n_pages
    table[2, 0], table[2, 6] = 2 ** 31 - 1, -2 ** 31
    table[4, 3::5] = n_pages + 3
    _run(new, lengths, 4, 2, d, 16, dtype, inputs=(q, kc, vc, table, cu, bits), tree=tree)


@pytest.mark.parametrize("dtype", sv.DTYPES)
def test_scores_from_far_apart(dtype):
    inputs = _inputs([9, 33, 4], [700, 700, 90], 4, 1, 64, 16, dtype, 900)
    q, kc = inputs[:2]
    kc *= torch.linspace(0.1, 3.0, len(kc))[:, None, None, None].to(dtype)
    kc[3, 5] = (4.0 * q[0, 1]).to(dtype)
    _run([9, 33, 4], [700, 700, 90], 4, 1, 64, 16, dtype, inputs=inputs)


@pytest.mark.parametrize("dtype", sv.DTYPES)
def test_shared_pages_slices_given_outputs_and_rows_of_no_sequence(dtype):
    new, lengths = [10, 10, 7], [100, 100, 75]
    _, kc, vc, table, cu, bits = _inputs([27], [112], 4, 2, 128, 16, dtype, 1000)
    table = table.expand(3, -1).contiguous()
    q = sv.normal(27, 4, 128, seed=1001, dtype=dtype)
    wide = torch.zeros(27, 9 * 128, dtype=dtype, device="cuda")
    wide[:, 128:5 * 128] = q.flatten(1).cuda()
    cu = sv.starts(new)
    out, lse = torch.empty(27, 4, 128, dtype=dtype, device="cuda"), torch.empty(27, 4, device="cuda")
    r = lss.lss_paged_attn_tree(wide[:, 128:5 * 128].unflatten(1, (4, 128)), kc.cuda(), vc.cuda(), table.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda(), cu.cuda(),
                                tree=bits.cuda(), out=out, lse=lse)
    assert r[0] is out and r[1] is lse
    want, want_lse, ob, lb = co.tree_attention(q, kc, vc, table, lengths, cu, bits)
    sv.check(out, want, ob, "out")
    sv.check(lse, want_lse, lb, "lse")
    # rows in front of the first sequence and behind the last
    inputs = list(_inputs([4, 6], [50, 60], 4, 2, 64, 16, dtype, 1010, more_rows=9))
    inputs[4] = inputs[4] + 3
    _run([4, 6], [50, 60], 4, 2, 64, 16, dtype, inputs=inputs)


@pytest.mark.parametrize("dtype", sv.DTYPES)
def test_the_same_bits_every_time_and_scratch_that_holds_anything(dtype):
    new, lengths = [3, 10, 40, 64], [3000, 10, 800, 4096]
    q, kc, vc, table, cu, bits = (x.cuda() for x in _inputs(new, lengths, 8, 2, 128, 32, dtype, 1100))
    n = torch.tensor(lengths, dtype=torch.int32).cuda()
    first = lss.lss_paged_attn_tree(q, kc, vc, table, n, cu, tree=bits)
    need = lss.lss_paged_attn_tree_workspace_bytes(len(q), 4, 8, 2, 128, table.shape[1] * 32, q.element_size())
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    for fill in (0, 255, 127, 1):
        ws.fill_(fill)
        for a, b in zip(lss.lss_paged_attn_tree(q, kc, vc, table, n, cu, tree=bits, workspace=ws), first):
            assert torch.equal(sv.bits(a), sv.bits(b))


@pytest.mark.parametrize("dtype", sv.DTYPES)
def test_one_drafted_token_is_the_attention_of_one_token(dtype):
    lengths = [1, 33, 700, 64, 2000]
    q, kc, vc, table, cu, bits = _inputs([1] * 5, lengths, 8, 2, 64, 16, dtype, 1200)
    want, want_lse, ob, lb = co.tree_attention(q, kc, vc, table, lengths, cu, None)
    n = torch.tensor(lengths, dtype=torch.int32).cuda()
    for got, got_lse in (lss.lss_paged_attn_decode(q.cuda(), kc.cuda(), vc.cuda(), table.cuda(), n), lss.lss_paged_attn_tree(q.cuda(), kc.cuda(), vc.cuda(), table.cuda(), n, cu.cuda())):
        sv.check(got, want, ob, "out")
        sv.check(got_lse, want_lse, lb, "lse")


def test_refusals_of_the_binding():
    z = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt, device="cuda")
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
    q, kc, table, lengths, cu = z(3, 4, 64), z(2, 16, 2, 64), i32(1, 2), i32(1), i32(2)
    for change, match in (({"tree": i32(3, 1)}, "tree must be"), ({"tree": z(2, 1, dt=torch.int64)}, "tree must be"), ({"tree": z(3, 0, dt=torch.int64)}, "tree must be"),
                          ({"cu_q": i32(3)}, "one entry more"), ({"cu_q": cu.long()}, "cu_q must be"), ({"q": z(3, 4, 64, dt=torch.float32)}, "cache's dtype"),
                          ({"lse": z(4, 3, dt=torch.float32)}, "output has shape"), ({"out": z(3, 4, 64, dt=torch.float32)}, "bfloat16"),
                          ({"tree": torch.zeros(3, 1, dtype=torch.int64)}, "tree must be"), ({"workspace": torch.zeros(4)}, "workspace must be")):
        with pytest.raises(ValueError, match=match):
            lss.lss_paged_attn_tree(**{**dict(q=q, k_cache=kc, v_cache=kc, block_table=table, lengths=lengths, cu_q=cu), **change})
    with pytest.raises(lss.LssError, match="LSS_ERR_RANGE"):
        lss.lss_paged_attn_tree(q, kc, kc, table, lengths, cu, max_len=33)
    with pytest.raises(lss.LssError, match="LSS_ERR_RANGE"):
        lss.lss_paged_attn_tree(q, kc, kc, table, lengths, cu, out=q)
