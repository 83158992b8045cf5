"""Another CTA's shared memory may be touched only once that CTA has begun. Read
from the sources: in every kernel that maps an address of another CTA, a barrier of
the cluster stands before the first such access, and what arrives at it early arrives at
the kernel's entry."""
import glob
import os
import re

import pytest

from paper_2609_34867_gb300 import build as B

BARRIER = r"cluster_sync\(\)|cluster_begun_wait\(\)|sync_all\(\)"


def _code(path):
    return re.sub(r"//[^\n]*|/\*.*?\*/", "", open(path).read(), flags=re.S)


def _kernels(code):
    """(name, body) of each __global__ function."""
    for m in re.finditer(r"__global__(?:\s+void|\s+__launch_bounds__\([^{;]*?\)(?=\s*\w+\())+\s+(\w+)\([^;{]*\)\s*\{", code):
        depth, i = 1, m.end()
        while depth:
            depth += {"{": 1, "}": -1}.get(code[i], 0)
            i += 1
        yield m.group(1), code[m.end():i]


def _without_lambdas(body):
    """The body without the definitions of its named lambdas, and the names of those that
    touch other CTAs' memory, by themselves or through others."""
    lambdas = {}
    while m := re.search(r"auto (\w+) = \[[^\]]*\]\([^)]*\)(?: -> \w+)? \{", body):
        depth, i = 1, m.end()
        while depth:
            depth += {"{": 1, "}": -1}.get(body[i], 0)
            i += 1
        lambdas[m.group(1)] = body[m.end():i]
        body = body[:m.start()] + body[i:]
    names = set()
    while more := {n for n, text in lambdas.items() if n not in names and re.search(_access(names), text)}:
        names |= more
    return body, names


def _access(names):
    return "|".join([r"mapa_shared\("] + [rf"\b{n}\(" for n in sorted(names)])


SOURCES = sorted(p for p in glob.glob(os.path.join(B.CSRC, "*.cu")) if "mapa_shared(" in _code(p))


@pytest.mark.parametrize("path", SOURCES, ids=[os.path.basename(p) for p in SOURCES])
def test_a_barrier_stands_before_the_first_access(path):
    seen = 0
    for name, body in _kernels(_code(path)):
        if "mapa_shared(" not in body:
            continue
        seen += 1
        rest, lambdas = _without_lambdas(body)
        access = re.search(_access(lambdas), rest)
        barrier = re.search(BARRIER, rest)
        assert access and barrier and barrier.start() < access.start(), name
        if "cluster_begun_wait()" in rest:
            arrive = rest.index("cluster_begun_arrive()")
            assert arrive < rest.index("pdl_wait()") and rest.count("cluster_begun_arrive()") == 1, name
            assert rest.count("cluster_begun_wait()") == 1, name
    assert seen
