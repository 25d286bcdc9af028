"""Order and convergence within a warp, which a run does not show: hardware keeps a warp's stores in
order and its lanes mostly together, the programming model promises neither without a warp barrier.  Votes
and shuffles meet, but order no memory.  Checked in the sources (no GPU)."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_08186_gb300", "csrc")


def _source(name):
    return re.sub(r"//[^\n]*|/\*.*?\*/", "", open(os.path.join(CSRC, name)).read(), flags=re.S)


def test_partial_rows_are_ordered_before_they_are_computed_again():
    # decode_tc_kernel: a row's partial is stored by several lanes, then again by exact_row's lanes
    src = _source("sfa_decode.cu")
    again = src.index("exact_row<DH>(")
    stored = src.rindex("pml[row] =", 0, again)
    assert "__syncwarp();" in src[stored:again]


def test_rows_are_ordered_before_they_are_settled():
    # settle_rows: rows stored by a lane each (the LSE too) are read by these lanes, then stored by the whole warp
    src = _source("packed.cuh")
    body = src[src.index("void settle_rows("):]
    read, vote, store = (body.index(x) for x in ("finite8(", "__ballot_sync(", "a.o[q0"))
    assert "__syncwarp();" in body[:read] and "__syncwarp();" in body[read:vote] and vote < store
