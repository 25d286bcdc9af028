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


# The TMEM accesses (.sync.aligned) need the whole warp.  Behind a condition that single lanes decide, the lanes meet
# at a warp barrier, vote or shuffle before the next one.
LANE = re.compile(r"\bif \((?:lane == 0|lead|store|rv|q4 \* 32 \+ rr < a\.M)\b")
MEET = r"__syncwarp|__any_sync|__all_sync|__ballot_sync|__shfl\w*_sync|named_bar_sync|__syncthreads"


def _warp_level(body):
    """For each lane-level condition, in the order of the source: the next thing of the whole warp."""
    for m in LANE.finditer(body):
        rest = body[m.end():]
        yield body[m.start():m.start() + 60], re.search(r"\b(" + MEET + r"|tmem_(?:ld|st)\w*)\(", rest)


def _softmax(name):
    src = _source(name)
    for kernel in ("fwd_packed_kernel(", "fwd_packed256_kernel(", "decode_tc_kernel("):
        if kernel in src:
            src = src[src.index(kernel):]
            return src[src.index("const uint32_t tl ="):src.rindex("tmem_dealloc")]
    raise AssertionError(name)


def _closing(src, at):
    depth = 0
    for i in range(at, len(src)):
        depth += (src[i] == "{") - (src[i] == "}")
        if depth == 0:
            return i
    raise AssertionError("unbalanced source")


def test_lanes_meet_before_tmem_accesses():
    for name in ("sfa_fwd_packed.cu", "sfa_fwd_packed256.cu", "sfa_decode.cu"):
        body = _softmax(name)
        found = list(_warp_level(body))
        assert len(found) >= 2, name
        for where, m in found:
            assert m is None or not m.group(1).startswith("tmem_"), (name, where)


def test_store_loops_end_with_a_barrier():
    # O leaves in a loop: load from TMEM, store what is a row's.  The next round's load is the whole warp's again
    for name, loop in (("sfa_fwd_packed.cu", "for (int c = 0; c < DH / 32; ++c)"),
                       ("sfa_fwd_packed256.cu", "for (int c = 0; c < PC / 32; ++c)"),
                       ("sfa_decode.cu", "for (int cc = 0; cc < DH / 32; ++cc) {\n        uint32_t o[32];\n        tmem_ld32(tO + cc * 32, o);\n        tmem_ld_wait();\n        if")):
        body = _softmax(name)
        at = body.index(loop)
        at = body.index("{", at)
        assert body[at:_closing(body, at)].rstrip().endswith("__syncwarp();"), name


def test_the_masks_of_shared_tiles_are_decided_by_the_entry():
    # `own` differs from lane to lane: it is no condition of a branch
    for name in ("sfa_fwd_packed.cu", "sfa_fwd_packed256.cu"):
        assert not re.search(r"\bown\s*[<>]|[<>]=?\s*own\b", _softmax(name)), name


def test_copies_land_before_a_cta_that_gave_up_exits():
    # a bounded wait that runs out ends the kernel's work, not its copies in flight
    src = _source("sfa_decode_paged.cu")
    leave = src.index("if (__syncthreads_or(!alive)) return;")
    assert "mbar_drain(&sm.full[brought % STAGES], (brought / STAGES) & 1);" in src[leave - 300:leave]
    src = _source("sfa_fwd_packed256.cu")
    producer = src[src.index("if (warp == 0) {"):src.index("} else if (warp == 1) {")]
    for bar in ("land(&sm.full[u % NSLOT], u / NSLOT);", "land(&sm.q_full[c], queries - 1);", "land(&sm.v_tail[k & 3], k >> 2);"):
        assert bar in producer[producer.rindex("tiles += T;"):], bar
