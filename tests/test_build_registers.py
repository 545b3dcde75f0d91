"""The build fails where the compiler gives the attention kernel another number of registers than its warps share out."""
import os
import re

import pytest

from paper_2411_05289_b200 import build

LOG = """ptxas info    : 0 bytes gmem
ptxas info    : Compiling entry function '_ZN7spechub21attention_join_kernelI6__halfLi64EEEvNS_13AttKernelArgsE' for 'sm_100a'
ptxas info    : Function properties for _ZN7spechub21attention_join_kernelI6__halfLi64EEEvNS_13AttKernelArgsE
    0 bytes stack frame, 0 bytes spill stores, 0 bytes spill loads
ptxas info    : Used 56 registers, used 1 barriers
ptxas info    : Compiling entry function '_ZN7spechub16attention_kernelI6__halfLi64EEEvNS_13AttKernelArgsENS_7AttMapsE' for 'sm_100a'
ptxas info    : Function properties for _ZN7spechub16attention_kernelI6__halfLi64EEEvNS_13AttKernelArgsENS_7AttMapsE
    192 bytes stack frame, 4 bytes spill stores, 12 bytes spill loads
ptxas info    : Used %d registers, used 1 barriers, 192 bytes cumulative stack size, 1600 bytes smem
ptxas info    : Function properties for _ZN7spechub8row_bitsERKNS_13AttentionArgsERKNS_8AttPieceEii
    0 bytes stack frame, 0 bytes spill stores, 0 bytes spill loads
"""


def wanted():
    return int(re.search(r"kLaunchRegs = (\d+)", open(os.path.join(build.CSRC, "spechub_attention.cuh")).read()).group(1))


def test_registers_are_read_by_kernel():
    assert sorted(build.registers_of(LOG % 168).values()) == [56, 168]


def test_only_the_number_that_is_shared_out_is_taken():
    build.check_registers("x/launch_attention.cu", LOG % wanted())
    build.check_registers("x/launch_cache.cu", LOG % 40)
    for log in (LOG % (wanted() - 8), LOG % 200, ""):
        with pytest.raises(RuntimeError, match="registers"):
            build.check_registers("x/launch_attention.cu", log)
