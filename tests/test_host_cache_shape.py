"""The sizes a paged cache may have, driven by a small host program under the undefined-behaviour sanitizer (CPU)."""
from test_host_rules import _run


def test_sizes_of_a_cache_are_checked_without_overflow(tmp_path):
    # (max_pages * page_size was made before max_pages was bounded: 2^60 pages of 16 overflow)
    _run(tmp_path, "cache_shape_check")
