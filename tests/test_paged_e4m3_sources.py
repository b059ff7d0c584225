"""What the sources of the paged cache say of memory that a kernel in front of them writes: a kernel of this library is resident, by programmatic
dependent launch, while the one in front of it still runs, and what it reads has been written in its lifetime.  Loads for memory that is
constant as long as the kernel lives (ld.global.nc, __ldg, and what the compiler may make of pointers that share nothing with others) promise
nothing about such memory."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2511_21759_b200", "csrc")
SOURCES = sorted(os.path.basename(p) for p in glob.glob(os.path.join(CSRC, "paged*.cu*")))


def code_of(name):
    return re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())


@pytest.mark.parametrize("name", SOURCES)
def test_nothing_is_read_as_if_it_were_constant(name):
    text = code_of(name)
    for word in ("__ldg", "ld.global.nc", "ldu.", "__restrict__"):
        assert word not in text, word
