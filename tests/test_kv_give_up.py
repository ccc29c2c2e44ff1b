"""What the attention kernel does when a bounded wait runs out, read from its
source (no GPU is made to wait in vain): a warp's lanes may read the CTA's flag
before and after another warp sets it, so whatever a branch takes from it is the
warp's vote. Else a warp could come apart before an instruction that all of its
lanes have to meet at, and wait there for ever."""

import os
import re

import pytest

from paper_2607_08565_gb300 import build_lib


@pytest.fixture(scope="module")
def source():
    text = open(os.path.join(build_lib.CSRC, "attention.cu")).read()
    return re.sub(r"//[^\n]*", "", text)  # without comments


def body(source, signature):
    at = source.index(signature)
    depth, i = 0, source.index("{", at)
    for j in range(i, len(source)):
        depth += {"{": 1, "}": -1}.get(source[j], 0)
        if depth == 0:
            return source[i:j + 1]


def test_the_flag_is_read_by_vote(source):
    assert re.search(r"return __any_sync\(kFull, [^;]*abort[^;]*\);", body(source, "bool stopped("))
    # the one other reader: a wait, after which the lanes go on alike
    inside = body(source, "void mbar_wait(")
    reads = len(re.findall(r"->abort(?! = )", source)) - len(re.findall(r"->abort\) = ", source))
    in_wait = len(re.findall(r"->abort(?! = )", inside)) - len(re.findall(r"->abort\) = ", inside))
    assert (reads, in_wait) == (2, 1)


def test_all_lanes_vote(source):
    """No vote under a condition on the lane: before it in an expression, or around it."""
    assert "stopped(" not in body(source, "void mbar_wait(")
    calls = [m.start() for m in re.finditer(r"\bstopped\(", source)][1:]  # (the first is its definition)
    assert len(calls) >= 5
    for at in calls:
        before = source[source.rindex("\n", 0, at):at]
        assert not re.search(r"lane|elect\(|held|mine", before), before
        depth = 0
        for i in range(at, -1, -1):  # the conditions that the call stands in
            depth += {"}": 1, "{": -1}.get(source[i], 0)
            if depth < 0:
                depth = 0
                line = source[source.rindex("\n", 0, i) + 1:i]
                if line.startswith(("__device__", "__global__")) or "[&]" in line:
                    break
                assert not re.search(r"\blane\b|elect\(|\bheld\b|\bmine\b", line), line


def test_a_wait_ends_with_the_warp_together(source):
    inside = body(source, "void mbar_wait(")
    assert inside.rstrip(" \n}").endswith("__syncwarp();") and "return;" not in inside


def test_what_is_in_flight_lands_before_the_memory_goes(source):
    """The pause comes after every warp has stopped issuing, and before the CTA frees what copies and products write."""
    kernel = body(source, "k_paged_attention(const")
    together, pause, free = kernel.rindex("__syncthreads();"), kernel.index("__nanosleep"), kernel.index("tcgen05.dealloc")
    assert together < kernel.index("stopped(") < pause < free
    assert "__nanosleep" not in body(source, "void copy_tiles(")
