"""Each way that the paged attention is launched, as the first call of its instance
in a process: nothing that a launch needs may hang on an earlier call of other sizes.
A fresh process per instance; each call is compared with the formula."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

HERE = os.path.dirname(os.path.abspath(__file__))

PROGRAM = """
import sys
sys.path[:0] = [{root!r}, {here!r}]
import torch
from paper_2609_34867_gb300 import build, p4q
from test_gpu_paged_attention import check, make, run
build.build()
dev = torch.device("cuda:0")
for lens, H, Hkv, dh, page, dt in {calls!r}:
    c = make(dev, lens, H, Hkv, dh, page, dt, seed=len(lens))
    check(c, *run(p4q, dev, c))
"""


def _fresh(calls):
    r = subprocess.run([sys.executable, "-c", PROGRAM.format(root=os.path.dirname(HERE), here=HERE, calls=calls)],
                       capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]


# the first call of an instance (type, dh, heads past 8 or not, pages from 16 or below), then others of it
@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("first", [
    [60],            # one tile: a cluster of one CTA
    [1] * 3,
    [120] * 200,     # a CTA for each of many units
    [700],           # clusters
    [20000],         # ranges
])
def test_first_call(first, dt):
    """Pages of 16 and of 8, groups of 16 and of 4 heads, dh 128 and 64: eight instances in one process."""
    _fresh([(lens, H, 1, dh, page, dt) for H in (16, 4) for dh in (128, 64) for page in (16, 8)
            for lens in (first, [33], [500, 20])])


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("H,Hkv,dh,page", [(40, 40, 128, 16), (32, 8, 128, 8), (12, 1, 64, 64), (16, 1, 128, 16)])
@pytest.mark.parametrize("cols", [1, 44, 200, 4000])
def test_tables_wider_than_the_lengths(p4q, dev, dt, H, Hkv, dh, page, cols):
    """The table's width decides how a call is split: the same sequences in tables of each width."""
    from test_gpu_paged_attention import check, make, run
    for lens in ([704], [1, 0, 65], [300, 704, 12, 500]):
        need = max((n + page - 1) // page for n in lens)
        c = make(dev, lens, H, Hkv, dh, page, dt, seed=cols, cols=max(cols, need))
        check(c, *run(p4q, dev, c))
