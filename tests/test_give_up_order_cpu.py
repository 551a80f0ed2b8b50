"""What a kernel does after a wait that ran out (CPU, the sources): MMAs issued before may still be writing tensor memory, so it goes back
only behind the pause that lets them and the copies land; freed before, another block's sums could lie there already."""
import glob
import os
import re

import pytest

from paper_2012_00596_b200 import build

FREE, PAUSE = r"\btmem_dealloc(_pair)?\(", r"while \(clock64\(\) - t0 < \d+ll\)"
FILES = sorted(f for f in glob.glob(os.path.join(build.CSRC, "*.cu")) if re.search(FREE, open(f).read()) and re.search(PAUSE, open(f).read()))


def test_the_kernels_with_tensor_memory_and_a_pause_are_found():
    assert len(FILES) >= 12


@pytest.mark.parametrize("path", FILES, ids=os.path.basename)
def test_tensor_memory_goes_back_behind_the_pause(path):
    text = open(path).read()
    frees, pauses = ([m.start() for m in re.finditer(what, text)] for what in (FREE, PAUSE))
    assert len(frees) == len(pauses)
    assert all(p < f for p, f in zip(pauses, frees)), os.path.basename(path)
