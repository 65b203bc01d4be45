"""Rows of a sequence from starts that may hold anything, driven by a small host program under the undefined-behaviour sanitizer (CPU)."""
from test_host_rules import _run


def test_rows_between_starts_that_hold_anything(tmp_path):
    # (min(next, rows) - start overflowed for a next start of -2^31: 2^31 - .. rows, or tiles below 0)
    _run(tmp_path, "starts_check")
