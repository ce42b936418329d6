"""Barriers in the kernels' sources: what is set up or met by some threads before others rely on it.  Both are races that hardware
usually hides, so the sources are looked at."""
import os

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2407_16207_b200", "csrc")


def source(name):
    return open(os.path.join(CSRC, name)).read()


def between(text, begin, end):
    assert text.count(begin) == 1, begin
    text = text[text.index(begin):]
    return text[:text.index(end)]


@pytest.mark.parametrize("name,begin,copy", [
    ("gsd_attn_tc.cuh", "int pre = 0;", "load_pieces(u, n, n"),                             # the producer warp's first copies
    ("gsd_attn_paged_rows.cu", "mbar_init(full + 8 * s, 1);", "issue(s, s, pages)"),
])
def test_lanes_that_copy_wait_for_the_lane_that_sets_the_barriers_up(name, begin, copy):
    part = between(source(name), begin, copy)
    assert "__syncwarp();" in part


@pytest.mark.parametrize("name", ["gsd_paged.cu", "gsd_attn_paged_rows.cu", "gsd_kv8.cu"])
def test_clusters_meet_without_the_aligned_forms(name):
    # those want a whole warp to come together, which nothing promises behind branches of single threads
    lines = [line for line in source(name).splitlines() if "barrier.cluster." in line]
    assert lines and not any(".aligned" in line for line in lines)
