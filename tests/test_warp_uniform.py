"""A warp's lanes leave a collective alike. The sampler's lists of candidates are given
up by a counter that other warps count on meanwhile: read by every lane for itself, lanes
that saw different counts would have left the others alone in the votes that follow. Read
from the source: one lane's reading goes to all."""
import os
import re

from paper_2609_34867_gb300 import build as B


def test_the_candidates_counter_is_read_by_one_lane():
    code = re.sub(r"//[^\n]*", "", open(os.path.join(B.CSRC, "p4q_sample.cu")).read())
    reads = [m.start() for m in re.finditer(r"\*reinterpret_cast<volatile uint32_t\*>\(&s\.sent\)", code)]
    shared = [m.end() for m in re.finditer(r"__shfl_sync\(0xFFFFFFFFu, (?=\*reinterpret_cast<volatile uint32_t\*>\(&s\.sent\), 0\))", code)]
    assert reads and reads == shared
    # any other reading stands behind a barrier: by one warp, for the counts that CTAs exchange
    plain = re.findall(r"[^\n]*[^&]\bs\.sent\b[^\n]*", code)
    assert all(re.search(r"s\.sent = 0;|put32_lanes\(&s\.cand_n\[rank\], s\.sent\)", line) for line in plain), plain
