"""What the compiler made of the kernels for several continuations (CPU)."""
import re

import pytest

import _asm

SOURCES = ["lss_tree.hip", "lss_pages.hip", "lss_beam.hip"]


@pytest.fixture(scope="module")
def code(tmp_path_factory):
    return _asm.assembly(tmp_path_factory.mktemp("asm"), SOURCES)


def test_no_kernel_keeps_a_register_in_scratch_memory(code):
    # (the selection has functions that are called, and as many threads as leave a lane 128 registers: an edit is soon one too many)
    seen = 0
    for source, text in code.items():
        for name, size, dynamic in re.findall(r"\.amdhsa_kernel (\S+).*?\.amdhsa_private_segment_fixed_size (\d+).*?\.amdhsa_uses_dynamic_stack (\d)", text, re.S):
            seen += 1
            assert (size, dynamic) == ("0", "0"), (source, name, size, dynamic)
    assert seen >= 16
