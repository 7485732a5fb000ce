"""What the kernel of large tiles of the 8-bit integer products does behind the compiler's back, read from the assembly of its source:
the accumulators are AGPRs by name and M0 is set for the LDS-direct loads, so nothing else may use either; and nothing is spilled."""
import os
import re
import subprocess

import pytest

from paper_2508_03984_amd import build


@pytest.fixture(scope="module")
def lines(tmp_path_factory):
    asm = tmp_path_factory.mktemp("i8") / "wide.s"
    flags = [f for f in build.compile_flags() if f not in ("-fPIC", "-shared")]
    subprocess.check_call([build.HIPCC] + flags + ["-x", "hip", "--cuda-device-only", "-S", os.path.join(build.CSRC, "oz2_i8_wide.hip"), "-o", str(asm)])
    return [line.strip() for line in asm.read_text().splitlines()]


def code(lines):
    return [line for line in lines if line and not line.startswith((";", ".", "//")) and not line.endswith(":")]


def test_only_the_mfmas_and_the_reads_after_a_tile_use_agprs(lines):
    used = [line for line in code(lines) if re.search(r"\ba(\d+|\[)", line.split(";")[0])]
    assert used
    for line in used:
        assert re.match(r"(v_mfma_i32_16x16x64_i8 a\[\w+:\w+\], v\[\d+:\d+\], v\[\d+:\d+\], (0|a\[\w+:\w+\])$|v_accvgpr_read_b32 v\d+, a\[\w+\]$)", line), line


def test_only_the_loads_use_m0(lines):
    text = code(lines)
    at = [i for i, line in enumerate(text) if re.search(r"\bm0\b", line)]
    assert at
    for i in at:
        assert re.match(r"s_mov_b32 m0, s\d+$", text[i]), text[i]
        assert text[i + 1] == "s_nop 0" or text[i + 1].startswith("v_add_u32 "), text[i: i + 3]
        assert text[i + 2].startswith("global_load_lds_dword"), text[i: i + 3]
    assert sum(line.startswith("global_load_lds_dword") for line in text) == len(at)


def test_nothing_is_spilled_to_memory(lines):
    assert not [line for line in code(lines) if line.startswith("scratch_")]
    sizes = [int(line.split()[-1]) for line in lines if ".private_segment_fixed_size:" in line]
    assert sizes and not any(sizes)
