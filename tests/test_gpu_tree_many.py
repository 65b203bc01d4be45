"""Attention of drafted tokens of many sequences: a launch in front counts them once, what a workgroup does to find its part grows no more."""
import pytest
import torch

from paper_2311_02382_amd import lss
import _continuations as co
import _serving as sv

pytestmark = pytest.mark.gpu


def _inputs(new, lengths, H, H_kv, d, dtype, seed, page=16, n_pages=300):
    """Sequences over pages that they share: of each its own choice"""
    gen = torch.Generator().manual_seed(seed)
    table = torch.randint(0, n_pages, (len(new), max(-(-n // page) for n in lengths)), generator=gen).int()
    q, kc, vc = sv.normal(sum(new), H, d, seed=seed + 1, dtype=dtype), sv.normal(n_pages, page, H_kv, d, seed=seed + 2, dtype=dtype), sv.normal(n_pages, page, H_kv, d, seed=seed + 3, dtype=dtype)
    return q, kc, vc, table, sv.starts(new)


def _check(new, lengths, H, H_kv, d, dtype, seed, max_len=None, some=29):
    q, kc, vc, table, cu = _inputs(new, lengths, H, H_kv, d, dtype, seed)
    B = len(new)
    out, lse = torch.full(q.shape, 7.0, dtype=dtype, device="cuda"), torch.full(q.shape[:2], 7.0, device="cuda")
    lss.lss_paged_attn_tree(q.cuda(), kc.cuda(), vc.cuda(), table.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda(), cu.cuda(), max_len=max_len, out=out, lse=lse)
    torch.cuda.synchronize()
    for b in sorted({0, 1, 63, 64, 65, 1023, 1024, 4095, 4096, B - 2, B - 1} & set(range(B)) | set(range(7, B, max(1, B // some))) | set(torch.tensor(lengths).topk(min(3, B))[1].tolist())):
        mine = slice(int(cu[b]), int(cu[b + 1]))
        want, want_lse, ob, lb = co.tree_attention(q[mine], kc, vc, table[b:b + 1], lengths[b:b + 1], torch.tensor([0, new[b]]), None, max_len)
        sv.check(out[mine], want, ob, f"out of sequence {b}")
        sv.check(lse[mine], want_lse, lb, f"lse of sequence {b}")


# on either side of what is counted in front, of a workgroup's threads and of batches of batches; sequences without rows; bounds on the lengths below and above what is cut
@pytest.mark.parametrize("dtype", sv.DTYPES)
@pytest.mark.parametrize("B", [64, 65, 255, 256, 257, 1023, 1024, 1025, 4097])
def test_number_of_sequences(dtype, B):
    lengths = [1 + (53 * b) % 500 for b in range(B)]
    _check([1] * B, lengths, 4, 2, 64, dtype, 10)                                        # no tile is cut
    lengths = [max(1, (53 * b) % 90) for b in range(B)]
    lengths[B // 3], lengths[B - 1] = 4000, 2500
    _check([1] * B, lengths, 4, 2, 64, dtype, 20)
    new = [(b * b) % 4 if b % 64 != 5 else 0 for b in range(B)]
    _check(new, [max(x, n) for x, n in zip(lengths, new)], 12, 3, 128, dtype, 30)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B", [256, 257, 700])
def test_many_rows_of_many_sequences(d, B):
    new = [5 + b % 9 for b in range(B)]
    lengths = [new[b] + (31 * b) % 300 for b in range(B)]
    _check(new, lengths, 8, 2, d, torch.bfloat16, 40)                                     # (tables of 320 tokens: no tile is cut)
    lengths[1], lengths[B // 2] = 3000, 4000
    _check(new, lengths, 8, 2, d, torch.bfloat16, 50)


def test_most_sequences_without_rows():
    B = 70000
    new, lengths = [0] * B, [3] * B
    for i, b in enumerate((0, 63, 64, 4095, 4096, 4097, 65535, 65536, B - 1)):
        new[b], lengths[b] = 1 + i, 30 + 170 * i
    for max_len in (None, 512):
        q, kc, vc, table, cu = _inputs(new, lengths, 4, 2, 64, torch.bfloat16, 60)
        out, lse = lss.lss_paged_attn_tree(q.cuda(), kc.cuda(), vc.cuda(), table.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda(), cu.cuda(), max_len=max_len)
        for b in (0, 63, 64, 4095, 4096, 4097, 65535, 65536, B - 1):
            mine = slice(int(cu[b]), int(cu[b + 1]))
            want, want_lse, ob, lb = co.tree_attention(q[mine], kc, vc, table[b:b + 1], lengths[b:b + 1], torch.tensor([0, new[b]]), None, max_len)
            sv.check(out[mine], want, ob, f"out of sequence {b}")
            sv.check(lse[mine], want_lse, lb, f"lse of sequence {b}")


def test_a_captured_call_follows_its_lengths_and_starts():
    B, H, H_kv, d = 600, 4, 2, 64
    first = ([1] * B, [max(1, (53 * b) % 90) for b in range(B)])
    first[1][5] = 4000
    new = [2 if b % 2 else 0 for b in range(B)]
    second = (new, [max(2, (71 * b) % 80) for b in range(B)])
    second[1][B - 1], second[1][301] = 3900, 1000
    q, kc, vc, table, _ = _inputs([1] * B, [4000] * B, H, H_kv, d, torch.bfloat16, 70)
    lengths, cu = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(B + 1, dtype=torch.int32, device="cuda")
    qd, kd, vd, td = q.cuda(), kc.cuda(), vc.cuda(), table.cuda()
    out, lse = torch.empty(B, H, d, dtype=torch.bfloat16, device="cuda"), torch.empty(B, H, device="cuda")
    ws = torch.empty(lss.lss_paged_attn_tree_workspace_bytes(B, B, H, H_kv, d, 4000), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        lss.lss_paged_attn_tree(qd, kd, vd, td, lengths, cu, max_len=4000, out=out, lse=lse, workspace=ws)
    for rows, n in (first, second, first, second):
        lengths.copy_(torch.tensor(n, dtype=torch.int32))
        cu.copy_(sv.starts(rows))
        ws.fill_(0x7f)
        graph.replay()
        torch.cuda.synchronize()
        eager = lss.lss_paged_attn_tree(qd, kd, vd, td, lengths, cu, max_len=4000)
        assert torch.equal(sv.bits(out), sv.bits(eager[0])) and torch.equal(sv.bits(lse), sv.bits(eager[1]))


def _time(B, max_len):
    q, kc, vc, table, cu = _inputs([1] * B, [max_len if b == 0 else 20 for b in range(B)], 8, 8, 128, torch.bfloat16, 80)
    args = [x.cuda() for x in (q, kc, vc, table, torch.tensor([max_len if b == 0 else 20 for b in range(B)], dtype=torch.int32), cu)]
    times = []
    for _ in range(6):
        start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        start.record()
        lss.lss_paged_attn_tree(*args, max_len=max_len)
        end.record()
        torch.cuda.synchronize()
        times.append(start.elapsed_time(end))
    return min(times[1:])


@pytest.mark.parametrize("max_len", [512, 800])
def test_time_grows_with_the_number_of_sequences(max_len):
    # (four times as many took eleven times as long: every workgroup went over all of them)
    assert _time(8192, max_len) < 8 * _time(2048, max_len)
