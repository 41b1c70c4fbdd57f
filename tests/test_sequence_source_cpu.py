"""What the sequence operators' sources have to keep that no run of theirs shows."""
import os
import re

from paper_2301_09266_amd import build

CSRC = os.path.dirname(build.LIB)


def text(name):
    return open(os.path.join(CSRC, name)).read()


def test_lanes_exchange_through_lds_between_fences():
    """A wave barrier orders no memory for the compiler: the only one stands between
    fences of the wave's scope, where the scan's lanes hand values to each other."""
    fence = r'__builtin_amdgcn_fence\(__ATOMIC_ACQ_REL, "wavefront"\);\s*'
    assert re.search(r"void wave_exchange\(\) \{\s*" + fence
                     + r"__builtin_amdgcn_wave_barrier\(\);\s*" + fence + r"\}",
                     text("seq_common.h"))
    for src in build.SEQ_SRCS + [os.path.join(CSRC, "seq_common.h")]:
        body = text(os.path.basename(src))
        assert body.count("__builtin_amdgcn_wave_barrier") == body.count("void wave_exchange"), src
    # before and after the reads, forward and back
    assert text("selective_scan.hip").count("wave_exchange();") == 4
