"""What the compiler made of the attention's forward kernels and of the cache's (CPU)."""
import re

import pytest

import _asm

SOURCES = ["lss_fwd.hip", "lss_fwd_bf16.hip", "lss_f32.hip", "lss_paged.hip", "lss_decode.hip", "lss_packed.hip"]


@pytest.fixture(scope="module")
def code(tmp_path_factory):
    return _asm.assembly(tmp_path_factory.mktemp("asm"), SOURCES)


def test_forward_kernels_keep_their_registers(code):
    # (the float forward of d = 64 with dropout had two in scratch memory; the float backward's kernels keep some there and are not meant)
    seen = 0
    for source, text in code.items():
        for name, size in re.findall(r"\.amdhsa_kernel (\S+).*?\.amdhsa_private_segment_fixed_size (\d+)", text, re.S):
            if "bwd" in name:
                continue
            seen += 1
            assert size == "0", (source, name, size)
    assert seen > 40
