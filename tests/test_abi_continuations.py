"""Host-side checks of the entry points for several continuations that need no GPU: bad arguments are refused before anything is launched."""
import pytest

from paper_2311_02382_amd import lss


@pytest.fixture(scope="module")
def lib():
    if not lss.LIB_PATH.exists():
        from paper_2311_02382_amd.build import build_library
        build_library(verbose=False)
    return lss.load()


# fake (never dereferenced) device addresses: every call below must fail in the host checks or be empty
def _append(lib, positions=0x4004, rows=3, k=0x1000):
    return lib.lss_paged_append_ex(k, 128, 0x2000, 128, 0x3000, 256, 0x4104, 0x5004, 0x6004, positions, rows, 2, 4, 2, 64, 2, 8, 16, 4, 0x7008, 64, 0, 0x8000, 0x9000, 0xa000, 0,
                                   None)


def _tree(lib, q=0x1000, qs=256, kc=0x2000, vc=0x3000, lengths=0x4004, table=0x5004, cu=0x5104, tree=0x5208, words=1, rows=5, B=2, H=4, H_kv=2, d=64, eb=2, n_pages=8,
          page=16, max_pages=4, max_len=64, ws=0, wn=0, out=0x6000, lse=0x7004):
    return lib.lss_paged_attn_tree(q, qs, kc, vc, lengths, table, cu, tree, words, rows, B, H, H_kv, d, eb, n_pages, page, max_pages, max_len, ws, wn, out, lse, None)


def _fork(lib, lengths=0x1004, table=0x2004, parents=0x3004, room=0x4004, held=0x5004, B=3, S=5, H_kv=2, d=64, eb=2, n_pages=8, page=16, max_pages=4, ws=0x10000, wn=1 << 20,
          kc=0x6000, vc=0x7000, table_out=0x8004, lengths_out=0x9004, missing=0xa004):
    return lib.lss_paged_fork(lengths, table, parents, room, held, B, S, H_kv, d, eb, n_pages, page, max_pages, ws, wn, kc, vc, table_out, lengths_out, missing, None)


def _compact(lib, lengths=0x1004, table=0x2004, cu=0x3004, kept=0x4004, n_kept=0x5004, most=4, B=3, H_kv=2, d=64, eb=2, n_pages=8, page=16, max_pages=4, kc=0x6000, vc=0x7000,
             lengths_out=0x9004):
    return lib.lss_paged_compact(lengths, table, cu, kept, n_kept, most, B, H_kv, d, eb, n_pages, page, max_pages, kc, vc, lengths_out, None)


def _select(lib, logits=0x1000, stride=100, scores=0x100004, finished=0x200001, end=2, B=2, K=3, V=100, N=4, eb=2, ws=0, wn=0, scores_out=0x300004, parents=0x400004,
            tokens=0x500004, finished_out=0x600001):
    return lib.lss_beam_select(logits, stride, scores, finished, end, B, K, V, N, eb, ws, wn, scores_out, parents, tokens, finished_out, None)


@pytest.mark.parametrize("change,code", [(dict(positions=0x4002), -4), (dict(rows=-1), -2), (dict(k=0), -1), (dict(rows=0), 0)])
def test_append_with_positions(lib, change, code):
    assert _append(lib, **change) == code
    assert code == 0 or "paged_append" in lss.lss_last_error()


@pytest.mark.parametrize("change,code", [
    (dict(d=96), -3), (dict(eb=3), -2), (dict(H=5), -2), (dict(H_kv=3), -2), (dict(H=0), -2), (dict(B=-1), -2), (dict(B=(1 << 24) + 1), -2), (dict(page=17), -2),
    (dict(n_pages=0), -2), (dict(max_pages=1 << 60), -2), (dict(max_len=65), -5), (dict(max_len=-1), -5), (dict(qs=200), -2), (dict(qs=257), -4), (dict(rows=-1), -2),
    (dict(rows=(1 << 22) + 1), -2), (dict(B=(1 << 21) + 1), -2), (dict(words=0), -2), (dict(words=1025), -2), (dict(q=0), -1), (dict(kc=0), -1), (dict(vc=0), -1), (dict(lengths=0), -1),
    (dict(table=0), -1), (dict(cu=0), -1), (dict(out=0), -1), (dict(lse=0), -1), (dict(q=0x1004), -4), (dict(vc=0x3008), -4), (dict(out=0x6004), -4), (dict(table=0x5002), -4),
    (dict(cu=0x5102), -4), (dict(tree=0x5204), -4), (dict(lse=0x7001), -4), (dict(ws=0x10008, wn=1 << 30), -4), (dict(max_pages=4096, max_len=65536, ws=0x10000, wn=100), -6),
    (dict(max_pages=4096, max_len=65536), -6), (dict(out=0x1010), -5), (dict(out=0x1000 + 0x9f0), -5), (dict(qs=1024, out=0x1000 + 4 * 0x800 + 0x1f0), -5),
    (dict(B=0), 0), (dict(rows=0), 0), (dict(rows=0, q=0, out=0, tree=0, words=0), 0)])
def test_tree(lib, change, code):
    assert lib.lss_set_workspace(None, 0) == 0
    assert _tree(lib, **change) == code
    assert code == 0 or "paged_attn_tree" in lss.lss_last_error()


@pytest.mark.parametrize("change,code", [
    (dict(d=32), -3), (dict(eb=1), -2), (dict(H_kv=0), -2), (dict(B=-1), -2), (dict(B=(1 << 20) + 1), -2), (dict(S=-1), -2), (dict(S=(1 << 20) + 1), -2), (dict(page=24), -2),
    (dict(n_pages=1 << 31), -2), (dict(max_pages=0), -2), (dict(lengths=0), -1), (dict(table=0), -1), (dict(parents=0), -1), (dict(kc=0), -1), (dict(vc=0), -1),
    (dict(table_out=0), -1), (dict(lengths_out=0), -1), (dict(missing=0), -1), (dict(kc=0x6008), -4), (dict(parents=0x3002), -4), (dict(room=0x4001), -4), (dict(held=0x5002), -4),
    (dict(missing=0xa001), -4), (dict(ws=0x10004), -4), (dict(wn=16), -6), (dict(ws=0, wn=0), -6),
    (dict(table_out=0x2004), -5), (dict(table_out=0x2004 + 4 * 12 - 4), -5), (dict(table_out=0x2004 - 4 * 20 + 4), -5), (dict(lengths_out=0x1004), -5), (dict(lengths_out=0x3004), -5),
    (dict(missing=0x4004 + 16), -5), (dict(missing=0x5004 + 28), -5)])
def test_fork(lib, change, code):
    assert lib.lss_set_workspace(None, 0) == 0
    assert _fork(lib, **change) == code and "paged_fork" in lss.lss_last_error()


@pytest.mark.parametrize("change,code", [
    (dict(d=32), -3), (dict(eb=1), -2), (dict(H_kv=0), -2), (dict(B=-1), -2), (dict(B=(1 << 18) + 1), -2), (dict(most=-1), -2), (dict(page=24), -2), (dict(n_pages=0), -2),
    (dict(lengths=0), -1), (dict(table=0), -1), (dict(cu=0), -1), (dict(kept=0), -1), (dict(n_kept=0), -1), (dict(lengths_out=0), -1), (dict(kc=0), -1), (dict(vc=0), -1),
    (dict(kc=0x6004), -4), (dict(kept=0x4002), -4), (dict(lengths_out=0x9002), -4), (dict(lengths_out=0x1004), -5), (dict(lengths_out=0x4004 + 44), -5), (dict(B=0), 0)])
def test_compact(lib, change, code):
    assert _compact(lib, **change) == code
    assert code == 0 or "paged_compact" in lss.lss_last_error()


@pytest.mark.parametrize("change,code", [
    (dict(eb=1), -2), (dict(B=-1), -2), (dict(K=0), -2), (dict(K=65), -2), (dict(V=0), -2), (dict(V=1 << 30), -2), (dict(N=0), -2), (dict(N=65), -2), (dict(B=1 << 20), -2),
    (dict(stride=99), -2), (dict(stride=1 << 33), -2), (dict(end=100), -5), (dict(end=-2), -5), (dict(end=-1), -5), (dict(end=-1, finished=0), -5), (dict(logits=0), -1),
    (dict(scores=0), -1), (dict(scores_out=0), -1), (dict(parents=0), -1), (dict(tokens=0), -1), (dict(logits=0x1001), -4), (dict(eb=4, logits=0x1002), -4), (dict(scores=0x100002), -4),
    (dict(tokens=0x500002), -4), (dict(ws=0x10004, wn=1 << 30), -4), (dict(V=50000, stride=50000), -6), (dict(V=50000, stride=50000, ws=0x10000, wn=64), -6),
    (dict(scores_out=0x100004), -5), (dict(tokens=0x1000 + 1196), -5), (dict(finished_out=0x200006), -5), (dict(B=0), 0)])
def test_select(lib, change, code):
    assert lib.lss_set_workspace(None, 0) == 0
    assert _select(lib, **change) == code
    assert code == 0 or "beam_select" in lss.lss_last_error()


def test_scratch(lib):
    tree, fork, select = lib.lss_paged_attn_tree_workspace_bytes, lib.lss_paged_fork_workspace_bytes, lib.lss_beam_select_workspace_bytes
    assert tree(64, 4, 32, 8, 128, 1 << 20, 2) > 0
    for bad in ((0, 4, 32, 8, 128, 4096, 2), (64, 0, 32, 8, 128, 4096, 2), (64, 4, 0, 8, 128, 4096, 2), (64, 4, 32, 5, 128, 4096, 2), (64, 4, 32, 8, 96, 4096, 2),
                (64, 4, 32, 8, 128, -1, 2), (64, 4, 32, 8, 128, 4096, 3), (1 << 20, 4, 32, 8, 128, 4096, 2)):
        assert tree(*bad) == 0
    assert fork(100, 7) >= 4 * (2 * 100 + 7) and fork(0, 7) == 0 and fork(100, -1) == 0
    assert select(2, 3, 100, 4) == 0 and select(2, 3, 50000, 4) > 0 and select(2, 17, 100, 4) > 0
    for bad in ((0, 3, 50000, 4), (2, 0, 50000, 4), (2, 65, 50000, 4), (2, 3, 50000, 65)):
        assert select(*bad) == 0
