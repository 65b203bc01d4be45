"""Scratch memory of the attention of drafted tokens: for tiles of rows whose keys are cut, of which there are few, whatever the number of rows, sequences and heads (CPU)."""
import itertools

import pytest

from paper_2311_02382_amd import lss


@pytest.fixture(scope="module")
def need():
    if not lss.LIB_PATH.exists():
        from paper_2311_02382_amd.build import build_library
        build_library(verbose=False)
    return lss.load().lss_paged_attn_tree_workspace_bytes


@pytest.mark.parametrize("eb", [2, 4])
@pytest.mark.parametrize("d", [64, 128])
def test_scratch_is_bounded(need, d, eb):
    # as many parts as three workgroups of 128 rows a compute unit, twice, at d = 64 (two at 128): sum of weight * value, maximum and sum in 32 bits each
    most = max(2 * 768 * 128 * (64 + 2), 2 * 512 * 128 * (128 + 2)) * 4 + (1 << 15)
    tried = 0
    for rows, B, (H, H_kv), max_len in itertools.product([1, 64, 8192, 65536, 1 << 19], [1, 48, 65, 1024, 65536, 1 << 19], [(1, 1), (32, 8), (32, 1), (64, 64)], [513, 8192, 1 << 30]):
        size = need(rows, B, H, H_kv, d, max_len, eb)
        if rows * H > 1 << 24 or B * H_kv > 1 << 22:
            assert size == 0
            continue
        tried += 1
        assert size <= most + 16 * (B // 64 + 2), (rows, B, H, H_kv, max_len, size)       # (and what is in front of every 64 sequences)
        assert size % 16 == 0
    assert tried > 200


def test_the_calls_that_asked_for_gigabytes(need):
    # 65536 and 4096 sequences of one token, 64 heads of keys; 1024 of 8 drafted tokens
    assert need(65536, 65536, 64, 64, 128, 8192, 2) <= 1 << 27
    assert need(4096, 4096, 64, 64, 128, 8192, 2) <= 1 << 27
    assert need(8192, 1024, 32, 8, 128, 8192, 2) <= 1 << 27
