"""Where lanes of a wavefront exchange values through LDS without a workgroup's barrier, the compiler may not keep a lane's own earlier values or
move its accesses: the scheduling barrier alone touches no memory in its eyes, so that a fence has to stand beside it (host only: the sources)."""
import os
import re

from paper_2601_02609_amd import build


def test_every_wave_barrier_has_its_fence():
    bare = []
    for name in sorted(os.listdir(build.CSRC)):
        with open(os.path.join(build.CSRC, name)) as source:
            lines = source.read().split("\n")
        for i, line in enumerate(lines):
            if "__builtin_amdgcn_wave_barrier" in line and not re.search(r'__builtin_amdgcn_fence\(__ATOMIC_ACQ_REL, "wavefront"', lines[i - 1]):
                bare.append(f"{name}:{i + 1}")
    assert not bare
