"""The barrier before another CTA's shared memory is touched, in kernels that headers hold (several
sources make kernels of one template). Read from the sources as in test_cluster_begin."""
import glob
import os
import re

from paper_2609_34867_gb300 import build as B
from test_cluster_begin import BARRIER, _access, _code, _kernels, _without_lambdas


def test_a_barrier_stands_before_the_first_access_in_headers():
    seen = []
    for path in sorted(glob.glob(os.path.join(B.CSRC, "*.cuh"))):
        for name, body in _kernels(_code(path)):
            if "mapa_shared(" not in body:
                continue
            seen.append(name)
            rest, lambdas = _without_lambdas(body)
            access, barrier = re.search(_access(lambdas), rest), re.search(BARRIER, rest)
            assert access and barrier and barrier.start() < access.start(), name
            if "cluster_begun_wait()" in rest:
                assert rest.index("cluster_begun_arrive()") < rest.index("pdl_wait()"), name
                assert rest.count("cluster_begun_arrive()") == rest.count("cluster_begun_wait()") == 1, name
    assert seen == ["paged_attention_kernel"]
