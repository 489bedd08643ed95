"""Lanes of a wave that hand values to one another through LDS without a block's barrier: what keeps the compiler from
moving a lane's loads over the others' stores is a pair of fences around the wave's barrier, which alone orders no memory."""
import glob
import os
import re

from conftest import ROOT

BARRIER = "__builtin_amdgcn_wave_barrier"


def sources():
    files = [f for f in sorted(glob.glob(os.path.join(ROOT, "paper_2609_37899_amd", "csrc", "*"))) if f.endswith((".hip", ".hpp"))]
    assert files
    for f in files:
        with open(f) as s:
            yield os.path.basename(f), [re.sub(r"//.*", "", x).strip() for x in s.read().split("\n")]


def test_waves_barriers_stand_between_fences():
    found, bare = 0, []
    for name, lines in sources():
        code = [(i + 1, x) for i, x in enumerate(lines) if x]
        for k, (line, x) in enumerate(code):
            if BARRIER not in x:
                continue
            found += 1
            before, behind = (code[j][1] if 0 <= j < len(code) else "" for j in (k - 1, k + 1))
            if not ("__builtin_amdgcn_fence(__ATOMIC_RELEASE, \"wavefront\")" in before
                    and "__builtin_amdgcn_fence(__ATOMIC_ACQUIRE, \"wavefront\")" in behind):
                bare.append(f"{name}:{line}")
    assert found and not bare, bare
