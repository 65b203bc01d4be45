"""The choice of a packed forward launch's form, driven by a small host program under the undefined-behaviour sanitizer (CPU)."""
from test_host_rules import _run


def test_packed_plan_takes_forms_there_is_a_kernel_for(tmp_path):
    _run(tmp_path, "packed_plan_check")
