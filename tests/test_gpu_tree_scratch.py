"""Attention of drafted tokens where a few of many tiles of rows are cut into parts: scratch memory is theirs alone."""
import pytest
import torch

from paper_2311_02382_amd import lss
import _continuations as co
import _serving as sv

pytestmark = pytest.mark.gpu


# a few long sequences among many short ones; rows of a tile: 16, 32, 128 in bf16
@pytest.mark.parametrize("dtype", sv.DTYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,n,H,H_kv", [(3, 2, 8, 8), (50, 1, 4, 4), (64, 5, 12, 4), (65, 6, 8, 2), (700, 1, 8, 8), (700, 5, 8, 2), (2000, 2, 4, 2)])
def test_few_tiles_are_cut(dtype, d, B, n, H, H_kv):
    new = [1 + (b * n) % n + (b % n) if n > 1 else 1 for b in range(B)]
    long = {0: 6000, B // 2: 9000, B - 1: 4100}
    lengths = [max(new[b], long.get(b, 3 + (7 * b) % 60)) for b in range(B)]
    table, n_pages = sv.tables(lengths, 16, B)
    gen = torch.Generator().manual_seed(B)
    q, kc, vc = sv.normal(sum(new), H, d, seed=6, dtype=dtype), sv.normal(n_pages, 16, H_kv, d, seed=7, dtype=dtype), sv.normal(n_pages, 16, H_kv, d, seed=8, dtype=dtype)
    bits, cu = torch.cat([co.random_tree(m, 1, gen) for m in new]), sv.starts(new)
    need = lss.lss_paged_attn_tree_workspace_bytes(len(q), B, H, H_kv, d, table.shape[1] * 16, q.element_size())
    guard = 1 << 16
    ws = torch.full((need + 2 * guard,), 0x7f, dtype=torch.uint8, device="cuda")
    for tree in (bits, None):
        out, lse = lss.lss_paged_attn_tree(q.cuda(), kc.cuda(), vc.cuda(), table.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda(), cu.cuda(),
                                           tree=None if tree is None else tree.cuda(), workspace=ws[guard:guard + need])
        torch.cuda.synchronize()
        assert bool((ws[:guard] == 0x7f).all()) and bool((ws[guard + need:] == 0x7f).all())
        for b in sorted({0, 1, 2, B // 2 - 1, B // 2, B // 2 + 1, B - 2, B - 1} & set(range(B)) | set(range(0, B, 97))):
            mine = slice(int(cu[b]), int(cu[b + 1]))
            want, want_lse, ob, lb = co.tree_attention(q[mine], kc, vc, table[b:b + 1], lengths[b:b + 1], torch.tensor([0, new[b]]), None if tree is None else bits[mine])
            sv.check(out[mine], want, ob, f"out of sequence {b}")
            sv.check(lse[mine], want_lse, lb, f"lse of sequence {b}")


def test_every_tile_is_cut_and_none():
    # as many parts as there is room for: sizes of a part just above and just below the number of rounds
    for B in (1, 2, 17, 100):
        for length in (513, 640, 768, 769, 1500):
            new, lengths = [9] * B, [length + b % 2 for b in range(B)]
            table, n_pages = sv.tables(lengths, 64, B)
            q, kc, vc = sv.normal(9 * B, 16, 64, seed=6), sv.normal(n_pages, 64, 4, 64, seed=7), sv.normal(n_pages, 64, 4, 64, seed=8)
            cu = sv.starts(new)
            out, lse = lss.lss_paged_attn_tree(q.cuda(), kc.cuda(), vc.cuda(), table.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda(), cu.cuda())
            for b in {0, B // 2, B - 1}:
                mine = slice(int(cu[b]), int(cu[b + 1]))
                want, want_lse, ob, lb = co.tree_attention(q[mine], kc, vc, table[b:b + 1], lengths[b:b + 1], torch.tensor([0, new[b]]), None)
                sv.check(out[mine], want, ob, f"out of sequence {b}")
                sv.check(lse[mine], want_lse, lb, f"lse of sequence {b}")


def test_very_many_sequences_over_shared_pages():
    # half a million tiles of rows, none or three of which are cut
    B, H, d = 8192, 64, 128
    gen = torch.Generator().manual_seed(3)
    kc, vc = sv.normal(60, 16, H, d, seed=1), sv.normal(60, 16, H, d, seed=2)
    table, q = torch.randint(0, 60, (B, 60), generator=gen).int(), sv.normal(B, H, d, seed=3)
    cu = torch.arange(B + 1, dtype=torch.int32)
    for long in ({}, {0: 960, 4000: 901, B - 1: 777}):
        lengths = [long.get(b, 1 + b % 37) for b in range(B)]
        out, lse = lss.lss_paged_attn_tree(q.cuda(), kc.cuda(), vc.cuda(), table.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda(), cu.cuda())
        for b in (0, 1, 63, 64, 4000, 4001, B - 2, B - 1):
            want, want_lse, ob, lb = co.tree_attention(q[b:b + 1], kc, vc, table[b:b + 1], lengths[b:b + 1], torch.tensor([0, 1]), None)
            sv.check(out[b:b + 1], want, ob, f"out of sequence {b}")
            sv.check(lse[b:b + 1], want_lse, lb, f"lse of sequence {b}")
