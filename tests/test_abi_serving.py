"""Host-side checks of the serving entry points that need no GPU: bad arguments are refused before anything is launched."""
import pytest

from paper_2311_02382_amd import lss


@pytest.fixture(scope="module")
def lib():
    if not lss.LIB_PATH.exists():
        from paper_2311_02382_amd.build import build_library
        build_library(verbose=False)
    return lss.load()


# fake (never dereferenced) device addresses: every call below must fail in the host checks or be empty
def _append(lib, k=0x1000, ks=128, v=0x2000, vs=128, q=0x3000, qs=256, cu=0x4004, lengths=0x5004, table=0x6004, rows=3, B=2, H=4, H_kv=2, d=64, eb=2,
            n_pages=8, page=16, max_pages=4, freq=0x7008, rot=64, kc=0x8000, vc=0x9000, q_rot=0xa000, k_rot=0):
    return lib.lss_paged_append(k, ks, v, vs, q, qs, cu, lengths, table, rows, B, H, H_kv, d, eb, n_pages, page, max_pages, freq, rot, 0, kc, vc, q_rot, k_rot, None)


def _decode(lib, q=0x1000, qs=256, kc=0x2000, vc=0x3000, lengths=0x4004, table=0x5004, B=2, H=4, H_kv=2, d=64, eb=2, n_pages=8, page=16, max_pages=4,
            max_len=64, ws=0, wn=0, out=0x6000, lse=0x7004):
    return lib.lss_paged_attn_decode(q, qs, kc, vc, lengths, table, B, H, H_kv, d, eb, n_pages, page, max_pages, max_len, ws, wn, out, lse, None)


def _packed(lib, q=0x1000, qs=256, k=0x2000, ks=128, v=0x3000, vs=128, cu_q=0x4004, cu_k=0x5004, rows_q=5, rows_k=7, B=2, H=4, H_kv=2, d=64, eb=2,
            ws=0, wn=0, out=0x6000, lse=0x7004):
    return lib.lss_packed_attn_fwd(q, qs, k, ks, v, vs, cu_q, cu_k, rows_q, rows_k, B, H, H_kv, d, eb, 1, ws, wn, out, lse, None)


@pytest.mark.parametrize("change,code", [
    (dict(d=32), -3), (dict(eb=1), -2), (dict(H_kv=0), -2), (dict(H=0), -2), (dict(B=-1), -2), (dict(rows=-1), -2), (dict(page=8), -2), (dict(page=48), -2),
    (dict(page=1 << 17), -2), (dict(n_pages=0), -2), (dict(n_pages=1 << 31), -2), (dict(max_pages=0), -2), (dict(max_pages=1 << 27), -2),
    (dict(max_pages=1 << 60), -2), (dict(ks=127), -2), (dict(ks=132), -4), (dict(vs=64), -2), (dict(qs=250), -2), (dict(qs=260), -4), (dict(rot=24), -2),
    (dict(rot=80), -2), (dict(rot=-16), -2), (dict(k=0), -1), (dict(v=0), -1), (dict(kc=0), -1), (dict(vc=0), -1), (dict(lengths=0), -1), (dict(table=0), -1),
    (dict(freq=0), -1), (dict(q_rot=0), -1), (dict(q=0), -1), (dict(k=0x1008), -4), (dict(kc=0x8004), -4), (dict(q_rot=0xa002), -4), (dict(k_rot=0xb008), -4),
    (dict(lengths=0x5002), -4), (dict(cu=0x4001), -4), (dict(freq=0x7004), -4), (dict(rows=(1 << 24) + 1), -2), (dict(ks=1 << 31), -2),
    (dict(H_kv=8192, ks=8192 * 128, vs=8192 * 128, d=128, rot=0, qs=512, page=1024), -2),
    (dict(rows=0), 0), (dict(B=0), 0), (dict(rows=0, k=0, kc=0, lengths=0), 0)])
def test_append(lib, change, code):
    assert _append(lib, **change) == code
    assert code == 0 or "paged_append" in lss.lss_last_error()


@pytest.mark.parametrize("change,code", [
    (dict(d=96), -3), (dict(eb=3), -2), (dict(H=5), -2), (dict(H_kv=3), -2), (dict(H=0), -2), (dict(B=-1), -2), (dict(B=(1 << 24) + 1), -2), (dict(page=17), -2),
    (dict(n_pages=-1), -2), (dict(max_len=65), -5), (dict(max_len=-1), -5), (dict(qs=200), -2), (dict(qs=257), -4), (dict(q=0), -1), (dict(kc=0), -1),
    (dict(vc=0), -1), (dict(lengths=0), -1), (dict(table=0), -1), (dict(out=0), -1), (dict(lse=0), -1), (dict(q=0x1004), -4), (dict(vc=0x3008), -4),
    (dict(out=0x6004), -4), (dict(table=0x5002), -4), (dict(lse=0x7001), -4), (dict(H=4096, H_kv=1, B=(1 << 11) + 1, qs=4096 * 64), -2),
    (dict(max_pages=4096, max_len=65536), -6), (dict(max_pages=4096, max_len=65536, ws=0x10000, wn=100), -6), (dict(ws=0x10008, wn=1 << 30), -4),
    (dict(B=0), 0), (dict(B=0, q=0, out=0), 0)])
def test_decode(lib, change, code):
    assert lib.lss_set_workspace(None, 0) == 0
    assert _decode(lib, **change) == code
    assert code == 0 or "paged_attn_decode" in lss.lss_last_error()


@pytest.mark.parametrize("change,code", [
    (dict(d=63), -3), (dict(eb=8), -2), (dict(H=3), -2), (dict(H_kv=0), -2), (dict(B=-1), -2), (dict(rows_q=-1), -2), (dict(rows_k=-1), -2), (dict(qs=255), -2),
    (dict(ks=100), -2), (dict(vs=129), -4), (dict(ks=136, eb=4), 1), (dict(q=0), -1), (dict(k=0), -1), (dict(v=0), -1), (dict(cu_q=0), -1), (dict(cu_k=0), -1),
    (dict(out=0), -1), (dict(lse=0), -1), (dict(k=0x2008), -4), (dict(out=0x6008), -4), (dict(cu_k=0x5002), -4), (dict(lse=0x7002), -4),
    (dict(rows_q=60, rows_k=9000), -6), (dict(rows_q=60, rows_k=9000, ws=0x10000, wn=1000), -6), (dict(ws=0x10004, wn=1 << 30), -4),
    (dict(rows_q=(1 << 27) + 1, H=8, qs=512), -2), (dict(B=(1 << 15) + 1, H_kv=128, H=128, ks=8192, vs=8192, qs=8192), -2),
    (dict(B=0), 0), (dict(rows_q=0), 0)])
def test_packed(lib, change, code):
    assert lib.lss_set_workspace(None, 0) == 0
    if code == 1:       # rows of float may be a multiple of 4 elements apart
        assert _packed(lib, **change, k=0x2008) == -4 and "tensor pointers" in lss.lss_last_error()
        return
    assert _packed(lib, **change) == code
    assert code == 0 or "packed_attn_fwd" in lss.lss_last_error()


def test_scratch_of_the_attention_of_one_token(lib):
    need = lib.lss_paged_attn_workspace_bytes
    assert need(4, 2, 64, 64) == 0 and need(4, 2, 64, 1 << 20) > 0
    assert need(32, 4, 128, 1 << 20) == need(32, 4, 128, 1 << 21) > need(16, 4, 128, 1 << 20)        # of the heads of a group, not of the lengths
    for bad in ((0, 1, 64, 4096), (4, 0, 64, 4096), (5, 2, 64, 4096), (4, 2, 96, 4096), (4, 2, 64, -1)):
        assert need(*bad) == 0


def test_scratch_of_packed_prompts(lib):
    need = lib.lss_packed_attn_workspace_bytes
    assert need(8192, 8192, 4, 32, 8, 128, 2) == 0                       # many rows: none
    assert need(60, 9000, 2, 4, 2, 64, 2) == 8 * 60 * 4 * 65 * 4         # eight splits' results and sums
    for bad in ((0, 9000, 2, 4, 2, 64, 2), (60, -1, 2, 4, 2, 64, 2), (60, 9000, 0, 4, 2, 64, 2), (60, 9000, 2, 5, 2, 64, 2), (60, 9000, 2, 4, 2, 32, 2),
                (60, 9000, 2, 4, 2, 64, 3)):
        assert need(*bad) == 0


def test_out_over_q_is_refused(lib):
    # decode: 2 rows of 4 heads of 64, 256 elements apart: 0x400 bytes from 0x1000; packed: 5 rows, 0xa00 bytes
    for call, end in ((_decode, 0x1400), (_packed, 0x1a00)):
        for out in (0x1000, 0x1010, end - 0x10, 0x1000 - (end - 0x1000) + 0x10):
            assert call(lib, out=out) == -5 and "out lies over q" in lss.lss_last_error()
    # rows further apart: 0x800 bytes from one to the next, the last one 0x200
    assert _decode(lib, qs=1024, out=0x19f0) == -5 and _packed(lib, qs=1024, out=0x31f0) == -5
