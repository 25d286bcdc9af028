"""Order and convergence within a warp of the 8-bit decoding kernels, which a run does not show (see test_warp_order_sources).
Checked in the sources (no GPU)."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_08186_gb300", "csrc")

# conditions that single lanes of a softmax warp decide; what brings the warp together again
LANE = re.compile(r"\bif \([^;{]*?\b(?:lane|key|column|vis)\b[^;{]*?\)")
MEET = r"__syncwarp|__(?:any|all|ballot)_sync|__shfl\w*_sync|__reduce_\w+_sync|named_bar_sync|group_any|note_losses"


def test_lanes_meet_before_they_access_tensor_memory():
    """The accesses (.sync.aligned) need the whole warp: behind a condition that single lanes decide comes a warp's meeting
    first, around a loop's end too."""
    src = open(os.path.join(CSRC, "sfa_decode_q8_tc.cu")).read()
    src = re.sub(r"//[^\n]*", "", src)
    body = src[src.index("const int wg = (warp - 2) >> 2"):src.rindex("tmem_dealloc")]
    loop = body[body.index("for (int hf = 0; hf < HV; ++hf) {\n          uint32_t o[3][16]"):]
    loop = loop[:loop.index("named_bar_sync")]
    seen = 0
    for text in (body, loop + loop):  # the loop over the head dim's halves begins with accesses
        for m in LANE.finditer(text):
            after = re.search(r"\b(?:(" + MEET + r")|tmem_(?:ld16|scale|ld_wait)\w*)\s*[(<]", text[m.end():])
            if after is not None:
                seen += 1
                assert after.group(1), text[m.start():m.end() + after.end()]
    assert seen > 10
