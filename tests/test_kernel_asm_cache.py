"""What the cache's kernels rest on in the code that the compiler makes of them for gfx950."""

import os
import re

import pytest

from paper_2511_23113_amd import build as b
from test_kernel_asm import asm_blocks, listing


def names_m0(line):
    return "m0" in re.split(r"[ ,\[\]]+", line.split(";")[0])


@pytest.mark.parametrize("source", ["cache_attn.hip", "cache_attn_long.hip", "cache_weights.hip"])
def test_m0_is_the_copies_own(source, tmp_path):
    # a copy to the LDS goes by M0, which its asm block (in cache_attn_long.hip one several sub-slots in front of it) sets and does not
    # say so: nothing else names it
    lines = listing(os.path.join(b.CSRC, source), str(tmp_path / "out.s"), b.EXTRA_FLAGS[source])
    set_here = sum(names_m0(line) for block in asm_blocks(lines) for line in block)
    copies = sum("global_load_lds_dwordx4" in line for block in asm_blocks(lines) for line in block)
    assert sum(map(names_m0, lines)) == set_here > 0 and copies > 0
    assert not [line for line in lines if re.match(r"(buffer|global)_load_lds", line) and "dwordx4" not in line]


def test_the_guard_sees_another_use_of_m0(tmp_path):
    # the same reading of a kernel in which the compiler itself needs M0: a copy by the builtin
    (tmp_path / "other.hip").write_text("""
#include <hip/hip_runtime.h>
__global__ void copies(const int* from, int* to) {
  __shared__ int there[64];
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(from + threadIdx.x), (__attribute__((address_space(3))) void*)there, 4, 0, 0);
  __syncthreads();
  to[threadIdx.x] = there[threadIdx.x];
}
""")
    lines = listing(str(tmp_path / "other.hip"), str(tmp_path / "other.s"))
    assert sum(map(names_m0, lines)) > 0 == sum(names_m0(line) for block in asm_blocks(lines) for line in block)
