"""CPU only: the ways that products grouped by expert take at the sizes of experts_cases.py, which are all that there are; the GPU tests check the
results there.  A constant of the estimate that moves a size to another way has to move the case, so that no way goes untested."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys

import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import experts_cases as cases  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CUTS = ("WIDE", "RING32", "RING128", "FEW128", "ANY32", "ANY64", "ANY128")
ENDS = ("", " tiles", " quarters", " small")


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")
def test_each_way_is_taken(tmp_path):
    exe = str(tmp_path / "experts_cut")
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2302_12445_amd", "csrc"),
                    os.path.join(ROOT, "tests", "native", "experts_cut.cpp"), "-o", exe], check=True)
    lines, wanted = [], []
    for counts, spare, outs, ins, dtype, *ways in cases.CASES:
        direct = cases.direct(counts, outs, ins, dtype)
        for kind, way in enumerate(ways):
            lines.append("%d %d %d %d %d %d %d %d\n" % (kind, dtype == "bf16", direct, sum(counts) + spare, len(counts), outs, ins,
                                                        cases.tiles(kind, counts, outs, ins)))
            wanted.append(((kind, dtype, direct), way))
    out = subprocess.run([exe], input="".join(lines), check=True, capture_output=True, text=True).stdout.splitlines()
    assert len(out) == len(wanted)
    reached = {key: set() for key in cases.WAYS}
    for line, said, (key, way) in zip(lines, out, wanted):
        cut, splits, end = map(int, said.split())
        got = CUTS[cut] + (" parts" if splits > 1 else "") + (" rounds" if end & 4 else "") + ENDS[end & 3]
        assert got == way, line
        reached[key].add(got)
    assert reached == cases.WAYS
