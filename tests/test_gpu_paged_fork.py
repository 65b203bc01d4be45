"""Sequences that take on their parents' pages, and accepted ones of drafted tokens: every element of tables and caches against the definition by lists."""
import pytest
import torch

from paper_2311_02382_amd import lss
import _continuations as co
import _serving as sv

pytestmark = pytest.mark.gpu


def _same(got, want, what):
    differ = sv.bits(got) != sv.bits(want)
    assert not bool(differ.any()), f"{what}: {int(differ.sum())} of {differ.numel()} values differ, first at {differ.nonzero()[0].tolist()}"


def _i32(x):
    return torch.tensor(x, dtype=torch.int32)


def _fork(table, lengths, parents, n_pages, page=16, H_kv=2, d=64, room=None, held=None, dtype=torch.bfloat16, seed=1):
    kc, vc = (sv.normal(n_pages, page, H_kv, d, seed=seed + i, dtype=dtype) for i in (0, 1))
    want = co.fork(kc, vc, table, lengths, parents, room, held)
    gk, gv, gt, gl = kc.cuda(), vc.cuda(), table.cuda(), _i32(lengths).cuda()
    got = lss.lss_paged_fork(gk, gv, gt, gl, _i32(parents).cuda(), room=None if room is None else _i32(room).cuda(), held=None if held is None else held.cuda())
    torch.cuda.synchronize()
    assert torch.equal(got[0].cpu(), want[2]), (got[0].cpu() != want[2]).nonzero()[:5]
    assert torch.equal(got[1].cpu(), want[3]) and int(got[2]) == want[4]
    _same(gk, want[0], "k_cache"), _same(gv, want[1], "v_cache")
    assert torch.equal(gt.cpu(), table) and gl.tolist() == lengths
    return got


@pytest.mark.parametrize("dtype", sv.DTYPES)
@pytest.mark.parametrize("page,H_kv,d", [(16, 2, 64), (64, 1, 128), (16, 5, 128)])
def test_beams(dtype, page, H_kv, d):
    # every place of a length in its page; parents once, twice, never, in any order
    lengths = [1, page - 1, page, page + 1, 3 * page, 3 * page + 5, 0, 2 * page + page // 2]
    table, n = sv.tables(lengths, page, 10, spare=30, extra=1)
    for seed, parents in enumerate(([0, 1, 2, 3, 4, 5, 6, 7], [5, 5, 5, 5, 1, 1, 7, 0], [7, 6, 5, 4, 3, 2, 1, 0], [3, 0, 3, 0, 3, 0], [2, 2, 4, 4, 4, 6, 6, 1, 1, 5, 7, 7, 7])):
        _fork(table, lengths, parents, n, page, H_kv, d, dtype=dtype, seed=20 + seed)


def test_beams_that_share_what_they_share():
    # beams of a prompt, step by step: the tables that one call leaves are the next one's, and every page is somebody's or free
    page, K, prompts = 16, 4, [5, 16, 40]
    gen = torch.Generator().manual_seed(3)
    table, used = sv.tables(prompts, page, 11, spare=0, extra=4)
    n, lengths, parents = 80, prompts, [b for b in range(3) for _ in range(K)]
    for step in range(40):
        got = _fork(table, lengths, parents, n, page, seed=30 + step)
        table, lengths = got[0].cpu(), got[1].tolist()
        assert int(got[2]) == 0
        if step % 13 == 12:
            lengths = [x - 1 for x in lengths]      # (a step that appends nothing)
        parents = [b * K + int(torch.randint(K, (), generator=gen)) for b in range(3) for _ in range(K)]
    # the prompts' full pages are shared still
    assert len(set(table[2 * K:, 0].tolist())) == 1 and len(set(table[2 * K:, 1].tolist())) == 1


def test_nobody_and_nothing():
    table, n = sv.tables([20, 33], 16, 12, extra=2)
    _fork(table, [20, 33], [-1, 1, 2, 2 ** 31 - 1, -2 ** 31, 0], n + 4, seed=40)
    _fork(table, [20, 33], [-1, -1], n, room=[40, 0], seed=41)                 # new sequences on the pages of those that are gone
    _fork(table, [20, 33], [], n, seed=42)
    _fork(table[:0], [], [0, -1], n, room=[3, 0], seed=43)
    _fork(table, [-7, 10 ** 9], [0, 1, 1], n + 9, room=[1, 1, 17], seed=44)        # lengths that are none and past the table


def test_room():
    page = 16
    lengths = [5, 16, 31, 100]
    table, n = sv.tables(lengths, page, 13, spare=60, extra=9)
    _fork(table, lengths, [0, 0, 1, 1, 2, 2, 3, 3], n, room=[0, 3, 0, 1, 100, 0, 12, 13], seed=50)        # (one that does not write reads: the writers move out)
    _fork(table, lengths, [0, 0, 0, 3], n, room=[0, 0, 0, 0], seed=51)
    _fork(table, lengths, [0, 0, 2, 2], n, room=[-5, 1, -2 ** 31, 2 ** 31 - 1], seed=52)


def test_too_few_pages():
    page, lengths = 16, [16, 20, 40]
    table, n = sv.tables(lengths, page, 14, spare=2, extra=1)
    got = _fork(table, lengths, [0, 0, 1, 1, 1, 2, 2], n, seed=60)
    assert int(got[2]) == 3
    got = _fork(table, lengths, [0, 1, 2], n, room=[10 ** 6, 2 ** 31 - 1, 1], seed=61)
    assert int(got[2]) > 10 ** 6 // 16


def test_too_few_pages_and_again():
    # what parents have is untouched by a call that had too few pages (only a sequence that is nobody's parent gives its own up): made again where there is room, it is whole
    page, lengths, parents = 16, [16, 20, 40, 70], [0, 0, 1, 1, 1, 2, 2]
    table, n = sv.tables(lengths, page, 21, spare=0, extra=1)
    kc, vc = (sv.normal(n + 8, page, 2, 64, seed=62 + i) for i in (0, 1))
    gk, gv, gt, gl, gp = kc.cuda(), vc.cuda(), table.cuda(), _i32(lengths).cuda(), _i32(parents).cuda()
    held = torch.zeros(n + 8, dtype=torch.int32)
    held[n:] = 1
    held[table[3].long()[:5]] = 1
    want = co.fork(kc, vc, table, lengths, parents, None, held)
    first = lss.lss_paged_fork(gk, gv, gt, gl, gp, held=held.cuda())
    assert int(first[2]) == want[4] > 0 and torch.equal(first[0].cpu(), want[2])
    for b in range(3):
        for nth in range(-(-lengths[b] // page)):
            rows = min(page, lengths[b] - nth * page)
            _same(gk[int(table[b, nth]), :rows], kc[int(table[b, nth]), :rows], "a parent's keys")
            _same(gv[int(table[b, nth]), :rows], vc[int(table[b, nth]), :rows], "a parent's values")
    want = co.fork(gk.cpu(), gv.cpu(), table, lengths, parents)
    again = lss.lss_paged_fork(gk, gv, gt, gl, gp)
    assert int(again[2]) == 0 == want[4] and torch.equal(again[0].cpu(), want[2]) and torch.equal(again[1].cpu(), want[3])
    _same(gk, want[0], "k_cache"), _same(gv, want[1], "v_cache")


def test_pages_that_others_hold():
    page, lengths = 16, [20, 33, 8]
    table, n = sv.tables(lengths, page, 15, spare=12, extra=2)
    held = torch.zeros(n, dtype=torch.int32)
    held[int(table[0, 0])], held[int(table[1, 2])] = 1, -7           # a full page, a partly filled one that even its one writer moves out of
    free = sorted(set(range(n)) - {int(x) for b, k in enumerate((2, 3, 1)) for x in table[b, :k]})
    held[free[0]], held[free[2]] = 2 ** 31 - 1, -2 ** 31
    got = _fork(table, lengths, [0, 1, 2, 2], n, held=held, seed=70)
    assert int(got[0][1, 2]) != int(table[1, 2]) and free[0] not in got[0].flatten().tolist()


def test_tables_with_anything_in_them():
    # numbers that are no page, the same page twice in a sequence and in two, as a full one and as a partly filled one
    table = _i32([[0, 1, 1, 9, -1], [1, -1, 2 ** 31 - 1, -2 ** 31, 3], [4, 4, 4, 4, 4], [1, 0, 5, 20, 0]])
    for seed, lengths in enumerate(([40, 70, 50, 20], [17, 33, 79, 64], [24, 12, 4, 70], [80, 80, 80, 80], [47, 48, 49, 16])):
        _fork(table, lengths, [0, 1, 2, 3], 20, seed=80 + seed)
        _fork(table, lengths, [3, 2, 1, 0, 0, 1, 2, 3], 20, room=[5, 0, 1, 30, 1, 2, 0, 16], seed=90 + seed)


def test_many_sequences_and_pages():
    # more sequences than the workgroup that deals out pages has threads, more pages than it looks at in one go, most of them taken
    gen = torch.Generator().manual_seed(5)
    page, B, S = 16, 700, 2600
    lengths = torch.randint(0, 200, (B,), generator=gen).tolist()
    table, n = sv.tables(lengths, page, 16, spare=20000, extra=2)
    held = (torch.rand(n, generator=gen) < 0.6).int()
    parents = torch.randint(-20, B, (S,), generator=gen).tolist()
    room = torch.randint(0, 40, (S,), generator=gen).tolist()
    _fork(table, lengths, parents, n, H_kv=1, seed=100)
    _fork(table, lengths, parents, n, H_kv=1, room=room, held=held, seed=101)


def test_long_tables():
    # tables of more pages than a workgroup has threads, large pages
    lengths = [16 * 600 + 3, 16 * 300, 50]
    table, n = sv.tables(lengths, 16, 17, spare=40, extra=700)
    _fork(table, lengths, [0, 1, 2, 0, 1], n, H_kv=1, seed=110)
    table, n = sv.tables([1000, 5000], 2048, 18, spare=5)
    _fork(table, [1000, 5000], [0, 1, 0, 1], n, page=2048, H_kv=3, seed=111)


def test_given_outputs_and_scratch_that_holds_anything():
    lengths = [20, 33, 8]
    table, n = sv.tables(lengths, 16, 19, spare=12, extra=2)
    kc, vc = (sv.normal(n, 16, 2, 64, seed=i) for i in (1, 2))
    want = co.fork(kc, vc, table, lengths, [2, 2, 0, 1])
    ws = torch.empty(lss.lss_paged_fork_workspace_bytes(n, 4), dtype=torch.uint8, device="cuda")
    for fill in (0, 255, 127):
        gk, gv = kc.cuda(), vc.cuda()
        outs = torch.empty(4, table.shape[1], dtype=torch.int32, device="cuda"), torch.empty(4, dtype=torch.int32, device="cuda"), torch.empty(1, dtype=torch.int32, device="cuda")
        ws.fill_(fill)
        for _ in range(2):                          # (what a call has done, it does again)
            r = lss.lss_paged_fork(gk, gv, table.cuda(), _i32(lengths).cuda(), _i32([[2, 2], [0, 1]]).cuda(), table_out=outs[0], lengths_out=outs[1], missing=outs[2], workspace=ws)
        assert all(a is b for a, b in zip(r, outs))
        assert torch.equal(outs[0].cpu(), want[2]) and torch.equal(outs[1].cpu(), want[3]) and int(outs[2]) == 0
        _same(gk, want[0], "k_cache"), _same(gv, want[1], "v_cache")


def _compact(new, lengths, kept, page=16, H_kv=2, d=64, dtype=torch.bfloat16, seed=1, table=None, n=None, wide=0, lists=None, counts=None):
    if table is None:
        table, n = sv.tables(lengths, page, seed, extra=1)
    kc, vc = (sv.normal(n, page, H_kv, d, seed=seed + i, dtype=dtype) for i in (1, 2))
    cu = sv.starts(new)
    want = co.compact(kc, vc, table, lengths, cu, kept)
    most = max([len(x) for x in kept] + [0]) + wide
    if lists is None:
        lists = torch.full((len(kept), most), 2 ** 31 - 1, dtype=torch.int32)
        for b, path in enumerate(kept):
            lists[b, :len(path)] = _i32(path)
    gk, gv, gl = kc.cuda(), vc.cuda(), _i32(lengths).cuda()
    got = lss.lss_paged_compact(gk, gv, table.cuda(), gl, cu.cuda(), lists.cuda(), _i32([len(x) for x in kept] if counts is None else counts).cuda())
    torch.cuda.synchronize()
    assert torch.equal(got.cpu(), want[2]), (got.cpu(), want[2])
    _same(gk, want[0], "k_cache"), _same(gv, want[1], "v_cache")
    assert gl.tolist() == lengths


@pytest.mark.parametrize("dtype", sv.DTYPES)
@pytest.mark.parametrize("page,H_kv,d", [(16, 2, 64), (64, 1, 128), (16, 17, 128), (32, 40, 128)])
def test_kept_tokens_move_to_the_front(dtype, page, H_kv, d):
    new = [10, 1, 64, 5, 0, 7, 33, 16]
    lengths = [10, 20, 100, 37, 12, 23, 33, 48]
    kept = [[0, 3, 4, 9], [0], [1, 2, 5, 11, 40, 41, 63], [], [], [0, 1, 2, 3, 4, 5, 6], [32], [2, 4, 6, 8, 10, 12, 14, 15]]
    for wide in (0, 3):
        _compact(new, lengths, kept, page, H_kv, d, dtype, seed=10, wide=wide)


def test_many_kept_tokens():
    gen = torch.Generator().manual_seed(6)
    new, lengths = [300, 129, 64, 700], [400, 129, 70, 5000]
    for share in (0.1, 0.5, 0.95, 1.0):
        kept = [[i for i in range(n) if torch.rand((), generator=gen) < share] for n in new]
        _compact(new, lengths, kept, seed=20)
    _compact([n % 9 for n in range(300)], [n % 9 + n % 50 for n in range(300)], [list(range(0, n % 9, 2)) for n in range(300)], seed=21)


def test_counts_and_numbers_that_are_none():
    # counts below 0, past the list and past what is drafted; numbers past what is drafted, below 0, below their place (those leave their place as it is)
    lists = _i32([[2, 5, 7, 8], [1, 3, 2, 4], [9, 10, 2 ** 31 - 1, 11], [-1, 3, -2 ** 31, 5]])
    new, lengths = [9, 3, 12, 6], [30, 3, 40, 16]
    _compact(new, lengths, [[], [1, 1, 2], [9, 10, 2, 11], [0, 3, 2, 5]], lists=lists, counts=[-3, 2 ** 31 - 1, 4, 100], seed=30)
    # fewer tokens than are drafted, lengths below 0 and past the table, no list at all
    _compact([9, 5, 6], [4, -3, 20], [[6, 8], [1], [5]], seed=31)
    _compact([4], [2 ** 31 - 1], [[1, 3]], table=_i32([[2, 0, 1]]), n=3, seed=32)
    _compact([4, 2], [10, 2], [[], []], seed=33)


def test_no_page_nothing_moves():
    table = _i32([[0, -1, 2], [9, 3, 2 ** 31 - 1], [4, -2 ** 31, 5]])
    _compact([20, 30, 40], [40, 33, 48], [[3, 5, 9, 13, 19], [0, 2, 12, 13, 14, 15, 16, 28, 29], [0, 9, 17, 30, 33, 39]], table=table, n=6, seed=40)


def test_refusals_of_the_binding():
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
    kc = torch.zeros(4, 16, 2, 64, dtype=torch.bfloat16, device="cuda")
    fork = dict(k_cache=kc, v_cache=kc.clone(), block_table=i32(2, 3), lengths=i32(2), parents=i32(4))
    compact = dict(k_cache=kc, v_cache=kc.clone(), block_table=i32(2, 3), lengths=i32(2), cu_q=i32(3), kept=i32(2, 4), n_kept=i32(2))
    for call, args, change, match in ((lss.lss_paged_fork, fork, dict(parents=i32(4).long()), "parents must be"), (lss.lss_paged_fork, fork, dict(room=i32(3)), "room must be"),
                                      (lss.lss_paged_fork, fork, dict(held=i32(3)), "held must have"), (lss.lss_paged_fork, fork, dict(table_out=i32(4, 2)), "output has shape"),
                                      (lss.lss_paged_fork, fork, dict(lengths=i32(3)), "disagree"), (lss.lss_paged_fork, fork, dict(parents=torch.zeros(4, dtype=torch.int32)), "parents must be"),
                                      (lss.lss_paged_compact, compact, dict(kept=i32(3, 4)), "a row for every sequence"), (lss.lss_paged_compact, compact, dict(n_kept=i32(3)), "a row for every"),
                                      (lss.lss_paged_compact, compact, dict(cu_q=i32(2)), "one entry more"), (lss.lss_paged_compact, compact, dict(kept=i32(4)), "kept must be"),
                                      (lss.lss_paged_compact, compact, dict(lengths_out=i32(2).long()), "torch.int32")):
        with pytest.raises(ValueError, match=match):
            call(**{**args, **change})
    with pytest.raises(lss.LssError, match="LSS_ERR_RANGE"):
        lss.lss_paged_fork(**{**fork, "parents": i32(2)}, table_out=fork["block_table"])
    with pytest.raises(lss.LssError, match="LSS_ERR_RANGE"):
        lss.lss_paged_compact(**compact, lengths_out=compact["lengths"])
