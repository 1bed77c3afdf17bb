"""What the paged attention's kernel rests on in the code that the compiler makes of it for gfx950."""

import os
import re

import pytest

from paper_2511_23113_amd import build as b
from test_kernel_asm import asm_blocks, listing
from test_kernel_asm_cache import names_m0


@pytest.fixture(scope="module")
def lines(tmp_path_factory):
    return listing(os.path.join(b.CSRC, "paged_attn.hip"), str(tmp_path_factory.mktemp("asm") / "paged.s"), b.EXTRA_FLAGS["paged_attn.hip"])


def test_m0_is_the_copies_own(lines):
    set_here = sum(names_m0(line) for block in asm_blocks(lines) for line in block)
    assert sum(map(names_m0, lines)) == set_here > 0
    for block in asm_blocks(lines):
        if any("_lds_" in line for line in block):      # each copy behind the setting of its destination, in one block
            assert re.match(r"s_mov_b32 m0, s\d+$", block[0]) and block[1] == "s_nop 0" and re.match(r"global_load_lds_dword(x4)? (v\[\d+:\d+\], off|v\d+, s\[\d+:\d+\])$", block[2])


def test_the_compiler_waits_for_no_memory_inside_the_loop(lines):
    # the copies are waited for by count, and the compiler does not know of them: a wait of its own in the loop over tiles would be one for all
    # that are under way.  The loop: between the wait in front of the next tile's copies and the wait for this one's
    own = [i for i, line in enumerate(lines) if lines[i - 1] == ";;#ASMSTART" and "vmcnt" in line and "vmcnt(0)" not in line]
    waits, ends = own[::2], own[1::2]
    assert len(waits) == len(ends) > 0
    for first, last in zip(waits, ends):
        assert first < last
        assert not [line for line in lines[first + 1:last] if "vmcnt" in line]
        # (by either of two ways: pages of the wave's keys each for itself, or one for all)
        assert sum("global_load_lds_dwordx4" in line for line in lines[first:last]) == 2 * int(re.search(r"vmcnt\((\d+)\)", lines[first])[1])
