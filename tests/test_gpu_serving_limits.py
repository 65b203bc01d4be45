"""The serving operators where their indices are large, their sequences many, and two calls run at once."""
import pytest
import torch

from paper_2311_02382_amd import lss
import _serving as sv
from test_gpu_paged_decode import _inputs, _want

pytestmark = pytest.mark.gpu


def _gpu(*tensors):
    return [t.cuda() for t in tensors]


def test_a_cache_whose_offsets_pass_32_bits():
    # over 2^32 elements a cache, 9 GB: tokens at both ends of it; appended, then attended to
    page, H_kv, d = 1024, 8, 128
    n_pages = 4300
    k_cache, v_cache = (torch.empty(n_pages, page, H_kv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    lengths = [1500, 700, 33]
    table = torch.tensor([[n_pages - 1, 0], [n_pages - 2, -1], [2049, -1]], dtype=torch.int32)
    rows = sum(lengths)
    q = sv.normal(3, 16, d, seed=1)
    k, v = (sv.normal(rows, H_kv, d, seed=i) for i in (2, 3))
    args = _gpu(table, torch.tensor(lengths, dtype=torch.int32))
    lss.lss_paged_append(k.cuda(), v.cuda(), k_cache, v_cache, *args, cu_seqlens=sv.starts(lengths).cuda())
    at = 0
    for b, n in enumerate(lengths):
        for i in range(0, n, page):
            m = min(page, n - i)
            for cache, rows_of in ((k_cache, k), (v_cache, v)):
                assert torch.equal(cache[int(table[b, i // page]), :m].cpu(), rows_of[at + i:at + i + m])
        at += n
    out, lse = lss.lss_paged_attn_decode(q.cuda(), k_cache, v_cache, *args)
    at = 0
    for b, n in enumerate(lengths):
        for g in range(H_kv):
            mine = slice(2 * g, 2 * g + 2)
            want, want_lse, ob, lb = sv.attention(q[b, mine], k[at:at + n, g], v[at:at + n, g], torch.full((2,), n), torch.bfloat16)
            sv.check(out[b, mine], want, ob, "out")
            sv.check(lse[b, mine], want_lse, lb, "lse")
        at += n


@pytest.mark.parametrize("dtype", sv.DTYPES)
@pytest.mark.parametrize("B,H,H_kv,d,longest", [(300, 8, 4, 64, 700), (150, 4, 4, 128, 900), (70, 20, 1, 64, 2000), (1, 1500, 1500, 64, 600), (3, 96, 2, 128, 1100)])
def test_more_sequences_and_heads_than_workgroups(dtype, B, H, H_kv, d, longest):
    lengths = [(331 * b + 17) % longest for b in range(B)]
    lengths[-1] = longest
    q, kc, vc, table = _inputs(lengths, H, H_kv, d, 16, dtype, 10 + B)
    out, lse = lss.lss_paged_attn_decode(*_gpu(q, kc, vc, table, torch.tensor(lengths, dtype=torch.int32)))
    some = sorted({0, 1, B // 2, B - 2, B - 1} & set(range(B)))
    want, want_lse, ob, lb = _want(q[some], kc, vc, table[some], [lengths[b] for b in some])
    sv.check(out[some], want, ob, "out")
    sv.check(lse[some], want_lse, lb, "lse")
    # every other sequence against itself alone
    for b in range(0, B, max(1, B // 9)):
        alone = lss.lss_paged_attn_decode(*_gpu(q[b:b + 1], kc, vc, table[b:b + 1], torch.tensor(lengths[b:b + 1], dtype=torch.int32)))
        _, _, ob, lb = _want(q[b:b + 1, :1], kc[:, :, :1], vc[:, :, :1], table[b:b + 1], lengths[b:b + 1]) if H <= 100 else (0, 0, None, None)
        if ob is not None:
            sv.check(out[b:b + 1, :1], alone[0][:, :1].double().cpu(), 2 * ob, f"sequence {b}")
            sv.check(lse[b:b + 1, :1], alone[1][:, :1].double().cpu(), 2 * lb, f"lse of sequence {b}")


def test_one_sequence_with_values_that_are_not_finite_is_alone_with_them():
    lengths = [700, 900, 40, 1300]
    q, kc, vc, table = _inputs(lengths, 8, 2, 64, 16, torch.bfloat16, 30)
    args = _gpu(q, kc, vc, table, torch.tensor(lengths, dtype=torch.int32))
    clean = lss.lss_paged_attn_decode(*args)
    args[1][int(table[1, 30]), 7, 0, 5] = float("nan")
    args[2][int(table[1, 3]), 2, 1, 9] = float("inf")
    got = lss.lss_paged_attn_decode(*args)
    for a, b in zip(got, clean):
        for i in (0, 2, 3):
            assert torch.equal(sv.bits(a[i]), sv.bits(b[i]))
    assert bool(torch.isnan(got[0][1, :4]).all()) and not bool(torch.isfinite(got[0][1, 4:, 9]).any())
    rest = torch.arange(64) != 9
    assert torch.equal(sv.bits(got[0][1, 4:][:, rest.cuda()]), sv.bits(clean[0][1, 4:][:, rest.cuda()]))


@pytest.mark.parametrize("dtype", sv.DTYPES)
def test_two_calls_at_once(dtype):
    # on two streams, with scratch of their own each, over and over
    calls = []
    for seed, (lengths, H, H_kv) in enumerate((([3000, 10, 800, 4096], 8, 2), ([900] * 20, 6, 3))):
        args = _gpu(*_inputs(lengths, H, H_kv, 128, 32, dtype, 40 + seed), torch.tensor(lengths, dtype=torch.int32))
        longest = args[3].shape[1] * 32
        ws = torch.empty(lss.lss_paged_attn_workspace_bytes(H, H_kv, 128, longest), dtype=torch.uint8, device="cuda")
        calls.append((lambda args=args, ws=ws: lss.lss_paged_attn_decode(*args, workspace=ws), torch.cuda.Stream()))
    for seed, (n_q, n_k, H, H_kv) in enumerate((([64], [4100], 8, 2), ([200, 31], [3000, 2500], 4, 2))):
        q, k, v = (sv.normal(sum(n), h, 64, seed=50 + 5 * seed + i, dtype=dtype).cuda() for i, (n, h) in enumerate(((n_q, H), (n_k, H_kv), (n_k, H_kv))))
        cu = sv.starts(n_q).cuda(), sv.starts(n_k).cuda()
        assert sv.packed_plan(sum(n_q), sum(n_k), len(n_q), H, H_kv, 64, dtype)[2] > 1
        ws = torch.empty(lss.lss_packed_attn_workspace_bytes(sum(n_q), sum(n_k), len(n_q), H, H_kv, 64, dtype.itemsize), dtype=torch.uint8, device="cuda")
        calls.append((lambda a=(q, k, v, *cu), ws=ws: lss.lss_packed_attn_fwd(*a, workspace=ws), torch.cuda.Stream()))
    want = [call() for call, _ in calls]
    torch.cuda.synchronize()
    got = [[] for _ in calls]
    for _ in range(12):
        for i, (call, stream) in enumerate(calls):
            with torch.cuda.stream(stream):
                got[i].append(call())
    torch.cuda.synchronize()
    for results, first in zip(got, want):
        for r in results:
            assert all(torch.equal(sv.bits(a), sv.bits(b)) for a, b in zip(r, first))


@pytest.mark.parametrize("dtype", sv.DTYPES)
def test_a_scratch_buffer_that_holds_anything(dtype):
    # what an earlier call of another kind left in it does not matter
    lengths = [3000, 1, 800, 0, 2000]
    args = _gpu(*_inputs(lengths, 4, 2, 64, 16, dtype, 60), torch.tensor(lengths, dtype=torch.int32))
    need = lss.lss_paged_attn_workspace_bytes(4, 2, 64, args[3].shape[1] * 16)
    first = None
    for fill in (0, 255, 127):
        ws = torch.full((need,), fill, dtype=torch.uint8, device="cuda")
        r = lss.lss_paged_attn_decode(*args, workspace=ws)
        first = first or r
        assert all(torch.equal(sv.bits(a), sv.bits(b)) for a, b in zip(r, first))
    with pytest.raises(ValueError, match="workspace of"):
        lss.lss_paged_attn_decode(*args, workspace=ws[:-16])


def test_starts_that_do_not_ascend_stay_within_the_tensors():
    # nothing is promised about the results: the rows around the outputs keep their values
    rows, H, H_kv, d = 200, 4, 2, 64
    q, k, v = (sv.normal(rows, h, d, seed=70 + h).cuda() for h in (H, H_kv, H_kv))
    for n, cu in enumerate(([0, 70, 30, 200], [200, 0, 500, -7], [-5, 300, 299, 0], [0] + [150, 20] * 40 + [200])):
        big_out = torch.full((rows + 64, H, d), 7.0, dtype=torch.bfloat16, device="cuda")
        big_lse = torch.full((H * rows + 1024,), 7.0, device="cuda")
        starts = torch.tensor(cu, dtype=torch.int32, device="cuda")
        lss.lss_packed_attn_fwd(q, k, v, starts, starts.flip(0).contiguous() if n % 2 else None, out=big_out[32:32 + rows], lse=big_lse[512:512 + H * rows].view(H, rows))
        k_cache, v_cache = (torch.full((12, 16, H_kv, d), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        B = len(cu) - 1
        table = torch.full((B, 3), 5, dtype=torch.int32, device="cuda")
        lss.lss_paged_append(k, v, k_cache[4:8], v_cache[4:8], table - 4, torch.full((B,), 40, dtype=torch.int32, device="cuda"), cu_seqlens=starts)
        torch.cuda.synchronize()
        assert bool((big_out[:32] == 7).all() and (big_out[32 + rows:] == 7).all() and (big_lse[:512] == 7).all() and (big_lse[512 + H * rows:] == 7).all())
        assert bool((k_cache[:5] == 7).all() and (k_cache[6:] == 7).all() and (v_cache[:5] == 7).all() and (v_cache[6:] == 7).all())
