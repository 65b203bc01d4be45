"""Starts of packed sequences at the ends of 32 bits, which do not ascend: nothing is promised of the results, but that nothing outside the tensors is read or written."""
import itertools

import pytest
import torch

from paper_2311_02382_amd import lss
import _continuations as co
import _serving as sv

pytestmark = pytest.mark.gpu

LOW, HIGH = -2 ** 31, 2 ** 31 - 1


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _guarded(*shape, dtype):
    n, guard = torch.Size(shape).numel(), 1 << 14
    whole = torch.full((n + 2 * guard,), 7, dtype=dtype, device="cuda")
    return whole[guard:guard + n].view(shape), lambda: bool((whole[:guard] == 7).all()) and bool((whole[guard + n:] == 7).all())


@pytest.mark.parametrize("dtype", sv.DTYPES)
@pytest.mark.parametrize("rows,H,H_kv,max_pages", [(24, 2, 2, 64), (60, 4, 2, 64), (60, 6, 2, 64), (200, 16, 2, 64), (200, 16, 2, 4)])
def test_drafted_tokens(dtype, rows, H, H_kv, max_pages):
    gen = torch.Generator().manual_seed(rows)
    q, kc, vc = sv.normal(rows, H, 64, seed=1, dtype=dtype), sv.normal(80, 16, H_kv, 64, seed=2, dtype=dtype), sv.normal(80, 16, H_kv, 64, seed=3, dtype=dtype)
    table = torch.randint(0, 80, (5, max_pages), generator=gen).int()
    lengths = [max_pages * 16, 40, 30, 50, max_pages * 16 - 7]
    need = lss.lss_paged_attn_tree_workspace_bytes(rows, 5, H, H_kv, 64, max_pages * 16, q.element_size())
    # (the first or the last sequence is in order; between them anything)
    for cu in ([0, 10, LOW, HIGH, LOW, rows], [0, 12, LOW, LOW, rows - 3, rows], [LOW, 20, LOW, HIGH, HIGH, LOW], [0, rows, LOW + 1, 5, HIGH, HIGH], [-1, rows // 2, LOW, rows, LOW, HIGH]):
        for fill in (0x77, 0x00, 0xff):
            out, out_ok = _guarded(rows, H, 64, dtype=dtype)
            lse, lse_ok = _guarded(rows, H, dtype=torch.float32)
            ws, ws_ok = _guarded(max(need, 16), dtype=torch.uint8)
            ws.fill_(fill)
            lss.lss_paged_attn_tree(q.cuda(), kc.cuda(), vc.cuda(), table.cuda(), _i32(lengths), _i32(cu), out=out, lse=lse, workspace=ws)
            torch.cuda.synchronize()
            assert out_ok() and lse_ok() and ws_ok(), (cu, fill)
    # no rows between starts that fall
    out, lse = lss.lss_paged_attn_tree(q.cuda(), kc.cuda(), vc.cuda(), table.cuda(), _i32(lengths), _i32([0, 20, LOW, LOW, LOW, LOW]))
    want, want_lse, ob, lb = co.tree_attention(q[:20], kc, vc, table[:1], lengths[:1], torch.tensor([0, 20]), None)
    sv.check(out[:20], want, ob, "out")
    sv.check(lse[:20], want_lse, lb, "lse")


@pytest.mark.parametrize("dtype", sv.DTYPES)
@pytest.mark.parametrize("rows,H,H_kv", [(24, 2, 2), (60, 6, 2), (300, 16, 2)])
@pytest.mark.parametrize("causal", [True, False])
def test_packed_sequences(dtype, rows, H, H_kv, causal):
    keys = 3 * rows
    q, k, v = sv.normal(rows, H, 64, seed=1, dtype=dtype), sv.normal(keys, H_kv, 64, seed=2, dtype=dtype), sv.normal(keys, H_kv, 64, seed=3, dtype=dtype)
    v[5, :, 3] = float("inf")                           # (rows are done once more over the keys that they see)
    kd, vd, qd = k.cuda(), v.cuda(), q.cuda()
    need = lss.lss_packed_attn_workspace_bytes(rows, keys, 3, H, H_kv, 64, q.element_size())
    starts_q = ([0, rows, LOW, HIGH], [0, LOW, HIGH, rows], [LOW, HIGH, LOW, rows])
    starts_k = ([0, keys, LOW, HIGH], [5, LOW, HIGH, LOW], [HIGH, LOW, LOW, 9], [LOW, keys - 1, LOW, HIGH])
    for cu_q, cu_k in itertools.product(starts_q, starts_k):
        out, out_ok = _guarded(rows, H, 64, dtype=dtype)
        lse, lse_ok = _guarded(H, rows, dtype=torch.float32)
        ws, ws_ok = _guarded(max(need, 16), dtype=torch.uint8)
        lss.lss_packed_attn_fwd(qd, kd, vd, _i32(cu_q), _i32(cu_k), causal=causal, out=out, lse=lse, workspace=ws)
        torch.cuda.synchronize()
        assert out_ok() and lse_ok() and ws_ok(), (cu_q, cu_k)
    # (rows are looked for among starts that ascend: with these some are not found, and not written)
    lss.lss_packed_attn_fwd(qd, kd, vd, _i32([0, rows, LOW]), _i32([5, LOW, HIGH]), causal=causal)
    # no keys between two starts that fall
    out, lse = lss.lss_packed_attn_fwd(qd, kd, vd, _i32([0, rows]), _i32([5, LOW]), causal=causal)
    assert bool((out == 0).all()) and bool((lse == -torch.inf).all())
