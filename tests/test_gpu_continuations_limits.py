"""The operators for several continuations at the ends of what they take: offsets past 32 bits, rows far apart, many sequences, arrays that hold anything."""
import pytest
import torch

from paper_2311_02382_amd import lss
import _continuations as co
import _serving as sv

pytestmark = pytest.mark.gpu


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.fixture(scope="module")
def far_cache():
    """Caches of more than 2^32 elements; a few pages at either end and in the middle hold values, the others anything"""
    page, H_kv, d = 1024, 8, 128
    n_pages = (1 << 32) // (page * H_kv * d) + 9
    kc, vc = (torch.empty(n_pages, page, H_kv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    pages = [0, 1, 2047, 2048, 2049, n_pages - 3, n_pages - 2, n_pages - 1]
    for i, p in enumerate(pages):
        kc[p], vc[p] = sv.normal(page, H_kv, d, seed=2 * i).cuda(), sv.normal(page, H_kv, d, seed=2 * i + 1).cuda()
    yield kc, vc, pages
    del kc, vc
    torch.cuda.empty_cache()


def _small(cache, table):
    """(cache of the pages that a table names, the table of their numbers there)"""
    used = sorted(set(table.flatten().tolist()))
    return cache[torch.tensor(used, device="cuda")].cpu(), torch.tensor([[used.index(x) for x in row] for row in table.tolist()], dtype=torch.int32)


@pytest.mark.parametrize("new", [[1, 2], [40, 7]])
def test_attention_over_pages_past_32_bits(far_cache, new):
    kc, vc, p = far_cache
    table = torch.tensor([[p[7], p[0], p[3]], [p[5], p[6], p[1]]], dtype=torch.int32)
    lengths, H = [2500, 1100], 16
    gen = torch.Generator().manual_seed(1)
    q, cu = sv.normal(sum(new), H, 128, seed=50), sv.starts(new)
    bits = torch.cat([co.random_tree(n, 1, gen) for n in new])
    out, lse = lss.lss_paged_attn_tree(q.cuda(), kc, vc, table.cuda(), _i32(lengths), cu.cuda(), tree=bits.cuda())
    k_small, at = _small(kc, table)
    v_small, _ = _small(vc, table)
    want, want_lse, ob, lb = co.tree_attention(q, k_small, v_small, at, lengths, cu, bits)
    sv.check(out, want, ob, "out")
    sv.check(lse, want_lse, lb, "lse")


def test_pages_past_32_bits_are_copied_and_compacted(far_cache):
    kc, vc, p = far_cache
    n_pages = len(kc)
    held = torch.ones(n_pages, dtype=torch.int32)
    held[p[7]], held[p[2]] = 0, 0                       # the only ones that are free
    table = _i32([[p[5], p[6]], [p[0], -1]])
    before = {x: (kc[x].clone(), vc[x].clone()) for x in p}
    got = lss.lss_paged_fork(kc, vc, table, _i32([1500, 100]), _i32([0, 0, 1, 1]), held=held.cuda())
    torch.cuda.synchronize()
    # (the pages that are shared are held by others too here: everybody moves out, and there are two pages for four)
    assert got[0].tolist() == [[p[5], p[2]], [p[5], p[7]], [-1, -1], [-1, -1]] and int(got[2]) == 2 and got[1].tolist() == [1501, 1501, 101, 101]
    for to in (p[2], p[7]):
        for c, i in ((kc, 0), (vc, 1)):
            assert torch.equal(sv.bits(c[to, :476]), sv.bits(before[p[6]][i][:476])) and torch.equal(sv.bits(c[to, 476:]), sv.bits(before[to][i][476:]))
    for x in (0, 1, 3, 4, 5, 6):
        assert torch.equal(sv.bits(kc[p[x]]), sv.bits(before[p[x]][0]))
    # compaction across the border of two far pages
    table = _i32([[p[6], p[7]]])
    old = kc[p[7]].clone()
    lengths = lss.lss_paged_compact(kc, vc, table, _i32([1040]), _i32([0, 30]), _i32([[5, 20, 29]]), _i32([3]))
    assert lengths.tolist() == [1013]
    assert torch.equal(sv.bits(kc[p[6], 1010]), sv.bits(before[p[6]][0][1015]))
    assert torch.equal(sv.bits(kc[p[6], 1011]), sv.bits(old[1010 + 20 - 1024])) and torch.equal(sv.bits(kc[p[6], 1012]), sv.bits(old[1010 + 29 - 1024]))


@pytest.mark.parametrize("dtype", sv.DTYPES)
def test_rows_far_apart(dtype):
    stride = 1 << 23
    wide = torch.empty(300 * stride, dtype=dtype, device="cuda")
    q = wide.as_strided((300, 4, 64), (stride, 64, 1))
    values = sv.normal(300, 4, 64, seed=1, dtype=dtype)
    q.copy_(values)
    new, lengths = [200, 100], [500, 400]
    table, n_pages = sv.tables(lengths, 16, 2)
    kc, vc = (sv.normal(n_pages, 16, 2, 64, seed=i, dtype=dtype) for i in (3, 4))
    cu = sv.starts(new)
    out, lse = lss.lss_paged_attn_tree(q, kc.cuda(), vc.cuda(), table.cuda(), _i32(lengths), cu.cuda())
    want, want_lse, ob, lb = co.tree_attention(values, kc, vc, table, lengths, cu, None)
    sv.check(out, want, ob, "out")
    sv.check(lse, want_lse, lb, "lse")


def test_logits_past_32_bits():
    stride = 1 << 27
    wide = torch.empty(40 * stride, dtype=torch.bfloat16, device="cuda")
    for V in (3001, 150001):
        logits = sv.normal(40, V, seed=V, std=3.0)
        rows = wide.as_strided((40, V), (stride, 1))
        rows.copy_(logits)
        scores = -5 * torch.rand(5, 8, generator=torch.Generator().manual_seed(V))
        want = co.select(logits, scores, 8)
        assert want[4] > 2 * co.LSE_BOUND
        got = lss.lss_beam_select(rows, scores.cuda(), 8)
        assert torch.equal(got[1].cpu().long(), want[1]) and torch.equal(got[2].cpu().long(), want[2])


@pytest.mark.parametrize("dtype", sv.DTYPES)
@pytest.mark.parametrize("long", [False, True])
def test_many_sequences_most_of_them_without_rows(dtype, long):
    B = 1500
    new, lengths = [0] * B, [3] * B
    for i, b in enumerate((0, 1, 63, 64, 65, 700, 1407, 1408, 1499)):
        new[b], lengths[b] = 1 + 5 * i, (700 if long else 90) + 7 * i
    table, n_pages = sv.tables(lengths, 16, 5)
    q, kc, vc = sv.normal(sum(new), 6, 64, seed=6, dtype=dtype), sv.normal(n_pages, 16, 2, 64, seed=7, dtype=dtype), sv.normal(n_pages, 16, 2, 64, seed=8, dtype=dtype)
    cu = sv.starts(new)
    for most in ((800,) if long else (160, 800)):
        out, lse = lss.lss_paged_attn_tree(q.cuda(), kc.cuda(), vc.cuda(), table.cuda(), _i32(lengths), cu.cuda(), max_len=min(most, table.shape[1] * 16))
        want, want_lse, ob, lb = co.tree_attention(q, kc, vc, table, lengths, cu, None, min(most, table.shape[1] * 16))
        sv.check(out, want, ob, "out")
        sv.check(lse, want_lse, lb, "lse")


def test_more_rows_than_the_launch_has_room_for_at_once():
    # many tiles of rows, which start with the longest sequences; as many sequences as that goes for, and more
    for B in (40, 70):
        new, lengths = [20 + b % 7 for b in range(B)], [30 + (211 * b) % 900 for b in range(B)]
        table, n_pages = sv.tables(lengths, 32, B)
        q, kc, vc = sv.normal(sum(new), 40, 64, seed=6), sv.normal(n_pages, 32, 20, 64, seed=7), sv.normal(n_pages, 32, 20, 64, seed=8)
        gen = torch.Generator().manual_seed(B)
        bits, cu = torch.cat([co.random_tree(n, 1, gen) for n in new]), sv.starts(new)
        out, lse = lss.lss_paged_attn_tree(q.cuda(), kc.cuda(), vc.cuda(), table.cuda(), _i32(lengths), cu.cuda(), tree=bits.cuda())
        some = [b for b in range(B) if b % 9 == 0]
        for b in some:
            mine = slice(int(cu[b]), int(cu[b + 1]))
            want, want_lse, ob, lb = co.tree_attention(q[mine], kc, vc, table[b:b + 1], lengths[b:b + 1], torch.tensor([0, new[b]]), bits[mine])
            sv.check(out[mine], want, ob, f"out of sequence {b}")
            sv.check(lse[mine], want_lse, lb, f"lse of sequence {b}")


@pytest.mark.parametrize("dtype", sv.DTYPES)
@pytest.mark.parametrize("rows,H,max_pages", [(60, 4, 4), (60, 4, 64), (200, 16, 64), (24, 2, 64)])
def test_starts_that_do_not_ascend_touch_nothing_else(dtype, rows, H, max_pages):
    # whatever the arrays hold: results lie between two guards, and the guards stay
    for cu in ([0, 50, 10, 60, 5, 70], [0, 60, 0, 60, 0, 60], [-5, 1000, -2 ** 31, 2 ** 31 - 1, 7, 3], [60, 40, 20, 10, 5, 0], [2 ** 31 - 1] * 6):
        gen = torch.Generator().manual_seed(rows)
        table = torch.randint(-2, 90, (5, max_pages), generator=gen).int()
        lengths = torch.tensor([2 ** 31 - 1, -7, 300, 17, 900], dtype=torch.int32)
        q, kc, vc = sv.normal(rows, H, 64, seed=1, dtype=dtype).cuda(), sv.normal(80, 16, 2, 64, seed=2, dtype=dtype).cuda(), sv.normal(80, 16, 2, 64, seed=3, dtype=dtype).cuda()
        guard = 4096
        out, lse = torch.full((2 * guard + rows * H * 64,), 7.0, dtype=dtype, device="cuda"), torch.full((2 * guard + rows * H,), 7.0, device="cuda")
        need = lss.lss_paged_attn_tree_workspace_bytes(rows, 5, H, 2, 64, max_pages * 16, q.element_size())
        ws = torch.full((need + 2 * guard,), 77, dtype=torch.uint8, device="cuda")
        bits = torch.randint(-2 ** 63, 2 ** 63 - 1, (rows, 1), generator=gen).cuda()
        for tree in (bits, None):
            lss.lss_paged_attn_tree(q, kc, vc, table.cuda(), lengths.cuda(), _i32(cu), tree=tree, out=out[guard:-guard].view(rows, H, 64), lse=lse[guard:-guard].view(rows, H),
                                    workspace=ws[guard:guard + need] if need else None)
            torch.cuda.synchronize()
        for x in (out, lse):
            assert bool((x[:guard] == 7.0).all()) and bool((x[-guard:] == 7.0).all())
        assert bool((ws[:guard] == 77).all()) and bool((ws[guard + need:] == 77).all())
