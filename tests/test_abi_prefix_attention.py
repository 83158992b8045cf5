"""Host-side checks of the entry point of shared prefixes (no GPU needed)."""
import ctypes

import pytest

from paper_2609_34867_gb300 import build as B
from test_abi_generation import BAD_CACHES, I, P, Paged, S, paged


@pytest.fixture(scope="module")
def lib():
    B.build()
    L = ctypes.CDLL(B.LIB)
    L.p4q_prefix_attention.argtypes = [P, I, I, ctypes.POINTER(Paged), P, P, P, I, ctypes.c_float, P, I, P, P, S, P]
    L.p4q_prefix_attention_workspace_bytes.argtypes = [I, I, I, I]
    L.p4q_prefix_attention_workspace_bytes.restype = S
    L.p4q_paged_attention_workspace_bytes.restype = S
    return L


def attend(lib, kv, q=16, ldq=1024, H=8, lens=4, start=4, prefix=4, groups=1, scale=0.1, o=16, ldo=1024, lse=None, ws=16,
           ws_bytes=1 << 30):
    return lib.p4q_prefix_attention(q, ldq, H, ctypes.byref(kv) if kv is not None else None, lens, start, prefix, groups,
                                    scale, o, ldo, lse, ws, ws_bytes, None)


@pytest.mark.parametrize("change,status", [(c, s) for c, s in BAD_CACHES if c != dict(dh=96)])
def test_cache_descriptions_are_checked(lib, change, status):
    assert attend(lib, paged(**change)) == status


@pytest.mark.parametrize("change,status", [
    (dict(H=0), 1), (dict(H=6), 1), (dict(scale=float("nan")), 1), (dict(scale=3e38), 1), (dict(groups=0), 1),
    (dict(groups=-1), 1), (dict(ldq=512), 1), (dict(ldo=512), 1), (dict(q=None), 1), (dict(lens=None), 1),
    (dict(start=None), 1), (dict(prefix=None), 1), (dict(o=None), 1), (dict(groups=3), 2),
    (dict(H=65536, ldq=1 << 24, ldo=1 << 24), 2), (dict(ldq=1028), 3), (dict(ldo=1028), 3), (dict(q=8), 3),
    (dict(o=24), 3), (dict(lens=2), 3), (dict(start=2), 3), (dict(prefix=6), 3), (dict(lse=2), 3), (dict(ws=None), 4),
    (dict(ws_bytes=1 << 20), 4), (dict(ws=8), 3),
])
def test_arguments_are_checked(lib, change, status):
    assert attend(lib, paged(), **change) == status


def test_more_rows_than_can_be_counted(lib):
    assert attend(lib, paged(seqs=1 << 20), H=4096, ldq=1 << 20, ldo=1 << 20) == 2


def test_missing_descriptions_and_empty_calls(lib):
    assert attend(lib, None) == 1
    none = paged(k=None, v=None, table=None, seqs=0)
    assert attend(lib, none, q=None, lens=None, start=None, prefix=None, groups=0, o=None, ws=None, ws_bytes=0) == 0


def test_workspace_grows_with_every_size(lib):
    size = lib.p4q_prefix_attention_workspace_bytes
    last = size(4, 1, 8, 64)
    assert last > 0
    assert size(5, 1, 8, 64) > last and size(4, 9, 8, 64) > last and size(4, 1, 9, 64) > last and size(4, 1, 8, 128) > last
    assert size(-1, 1, 8, 64) == 0 and size(4, 1, 0, 64) == 0 and size(4, 1, 8, 256) == 0
