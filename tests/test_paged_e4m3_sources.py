"""What the sources of the paged cache say, of memory that others write for the most part.

Of the kernel in front: a kernel of this library is resident, by programmatic
dependent launch, while the one in front of it still runs, and what it reads has been written in its lifetime.  Loads for memory that is
constant as long as the kernel lives (ld.global.nc, __ldg, and what the compiler may make of pointers that share nothing with others) promise
nothing about such memory.

Of other threads: the arrival that follows a thread's asynchronous copies (cp.async.mbarrier.arrive) is made when they have landed and orders
nothing that the thread has stored itself.

And of a call that has one wave of CTAs: what its shares are at least as long as all places have work decides nothing."""
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


@pytest.mark.parametrize("name", ["paged_e4m3_attention.cu", "paged_e4m3_attention_tc.cu"])
def test_a_scale_that_a_lane_writes_itself_is_followed_by_its_own_arrival(name):
    text = code_of(name)
    stores = [m.end() for m in re.finditer(r"\*scale = 1\.f;", text)]
    assert len(stores) == 1
    then = re.search(r"\b(mbar_arrive|copies_arrive)\(", text[stores[0]:])
    assert then.group(1) == "mbar_arrive"


@pytest.mark.parametrize("name", ["paged_e4m3_attention.cu", "paged_e4m3_attention_tc.cu"])
def test_one_wave_of_equal_shares_has_no_numbers_without_effect(name):
    calls = re.findall(r"paged_find_start<[^>]*>\(a, [^;]*?, (\d+), (\w+(?: \+ \d+)?), (\w+), start\);", code_of(name))
    assert calls and all(waves == "1" and full == "0" for waves, _, full in calls), calls
