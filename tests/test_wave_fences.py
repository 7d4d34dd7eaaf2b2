"""Lanes that hand values to each other in LDS meet behind a fence: the wave barrier alone does not keep the compiler from
moving an LDS access across it.  Read off the sources."""

import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2606_31145_amd", "csrc")
FENCE = re.compile(r'__builtin_amdgcn_fence\(__ATOMIC_ACQ_REL, "wavefront"\);\s*$')


def test_wave_barriers_stand_behind_a_fence():
    found = 0
    for path in sorted(glob.glob(os.path.join(CSRC, "*"))):
        with open(path) as f:
            pieces = f.read().split("__builtin_amdgcn_wave_barrier")
        for before in pieces[:-1]:
            assert FENCE.search(before), f"{os.path.basename(path)}:{before.count(chr(10)) + 1}"
            found += 1
    assert found
