"""Host-side checks of the generation operators' entry points (no GPU needed):
what is refused is refused before anything is launched."""
import ctypes

import pytest

from paper_2609_34867_gb300 import build as B

P, I, S = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t


class Paged(ctypes.Structure):
    _fields_ = [("k", P), ("v", P), ("table", P), ("page_stride", ctypes.c_int64), ("token_stride", ctypes.c_int64),
                ("head_stride", ctypes.c_int64), ("dtype", ctypes.c_int32), ("pages", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("Hkv", ctypes.c_int32), ("dh", ctypes.c_int32),
                ("seqs", ctypes.c_int32), ("table_ld", ctypes.c_int32), ("table_cols", ctypes.c_int32)]


@pytest.fixture(scope="module")
def lib():
    B.build()
    L = ctypes.CDLL(B.LIB)
    L.p4q_rope_append.argtypes = [P, I, P, I, P, I, I, I, P, P, I, I, I, P, P, P, ctypes.POINTER(Paged), P, I, P, I, P]
    L.p4q_paged_attention.argtypes = [P, I, I, ctypes.POINTER(Paged), P, ctypes.c_float, P, I, P, P, S, P]
    L.p4q_paged_attention_workspace_bytes.argtypes = []
    L.p4q_paged_attention_workspace_bytes.restype = S
    L.p4q_sample.argtypes = [P, I, ctypes.c_int64, I, I, P, P, P, P, P, P, P, P]
    return L


def paged(**changes):
    """A cache of 16 pages of 16 slots, 4 heads of 128, two sequences of 8 pages."""
    v = dict(k=16, v=16, table=4, page_stride=16 * 4 * 128, token_stride=4 * 128, head_stride=128, dtype=0, pages=16,
             page_size=16, Hkv=4, dh=128, seqs=2, table_ld=8, table_cols=8)
    v.update(changes)
    return Paged(**v)


BAD_CACHES = [
    (dict(k=None), 1), (dict(v=None), 1), (dict(table=None), 1), (dict(pages=-1), 1), (dict(page_size=0), 1),
    (dict(Hkv=0), 1), (dict(dh=0), 1), (dict(seqs=-1), 1), (dict(table_ld=7), 1), (dict(table_cols=-1, table_ld=0), 1),
    (dict(page_stride=0), 1), (dict(token_stride=64), 1), (dict(head_stride=-128), 1),
    (dict(dtype=2), 2), (dict(dtype=3), 2), (dict(page_size=24), 2), (dict(page_size=1 << 17), 2), (dict(dh=96), 1),
    (dict(dh=96, page_stride=8192, token_stride=512, head_stride=128), 2), (dict(Hkv=65536), 2),
    (dict(page_stride=8196), 3), (dict(token_stride=516), 3), (dict(head_stride=132), 3), (dict(k=8), 3),
    (dict(v=24), 3), (dict(table=2), 3),
]


def append(lib, kv, q=16, ldq=1024, k=16, ldk=512, v=16, ldv=512, T=2, H=8, cos=16, sin=16, max_pos=64, rot=128,
           inter=0, pos=4, rot_pos=None, seq=None, q_out=16, ldqo=1024, k_out=None, ldko=0):
    return lib.p4q_rope_append(q, ldq, k, ldk, v, ldv, T, H, cos, sin, max_pos, rot, inter, pos, rot_pos, seq,
                               ctypes.byref(kv) if kv is not None else None, q_out, ldqo, k_out, ldko, None)


def attend(lib, kv, q=16, ldq=1024, H=8, lens=4, scale=0.1, o=16, ldo=1024, lse=None, ws=16, ws_bytes=1 << 30):
    return lib.p4q_paged_attention(q, ldq, H, ctypes.byref(kv) if kv is not None else None, lens, scale, o, ldo, lse,
                                   ws, ws_bytes, None)


@pytest.mark.parametrize("change,status", BAD_CACHES)
def test_cache_descriptions_are_checked(lib, change, status):
    if change.get("dh") == 96 and "page_stride" not in change:
        change = dict(change, head_stride=64)  # a stride below dh
    assert append(lib, paged(**change)) == status
    assert attend(lib, paged(**change)) == status


@pytest.mark.parametrize("change,status", [
    (dict(T=-1), 1), (dict(H=0), 1), (dict(max_pos=0), 1), (dict(rot=0), 1), (dict(ldq=1016), 1), (dict(ldk=504), 1),
    (dict(ldv=504), 1), (dict(ldqo=512), 1), (dict(k_out=16, ldko=256), 1), (dict(q=None), 1), (dict(k=None), 1),
    (dict(v=None), 1), (dict(cos=None), 1), (dict(sin=None), 1), (dict(pos=None), 1), (dict(q_out=None), 1),
    (dict(T=3), 1),  # more tokens than sequences, and no seq
    (dict(rot=24), 2), (dict(rot=144), 2), (dict(H=65536, ldq=1 << 24, ldqo=1 << 24), 2),
    (dict(ldq=1028), 3), (dict(ldk=516), 3), (dict(ldv=516), 3), (dict(ldqo=1028), 3), (dict(k_out=16, ldko=516), 3),
    (dict(q=8), 3), (dict(k=8), 3), (dict(v=8), 3), (dict(cos=8), 3), (dict(sin=4), 3), (dict(q_out=2), 3),
    (dict(k_out=8, ldko=512), 3), (dict(pos=2), 3), (dict(rot_pos=1), 3), (dict(seq=6), 3),
])
def test_rope_append_validates_arguments(lib, change, status):
    assert append(lib, paged(), **change) == status


def test_rope_append_of_nothing_is_a_no_op(lib):
    assert append(lib, paged(), T=0) == 0
    assert append(lib, paged(k=None, v=None, table=None), T=0, q=None, k=None, v=None, pos=None, q_out=None) == 0
    assert append(lib, None, T=0) == 1


@pytest.mark.parametrize("change,status", [
    (dict(H=0), 1), (dict(H=6, ldq=768, ldo=768), 1), (dict(scale=float("nan")), 1), (dict(scale=float("inf")), 1),
    (dict(ldq=1016), 1), (dict(ldo=512), 1), (dict(q=None), 1), (dict(lens=None), 1), (dict(o=None), 1),
    (dict(H=65536 * 4, ldq=1 << 28, ldo=1 << 28), 2),
    (dict(ldq=1028), 3), (dict(ldo=1028), 3), (dict(q=8), 3), (dict(o=8), 3), (dict(lens=2), 3), (dict(lse=2), 3),
    (dict(ws=8), 3), (dict(ws=None), 4), (dict(ws_bytes=8), 4),
])
def test_paged_attention_validates_arguments(lib, change, status):
    assert lib.p4q_paged_attention_workspace_bytes() > 8
    assert attend(lib, paged(), **change) == status


def test_paged_attention_of_nothing_is_a_no_op(lib):
    assert attend(lib, paged(seqs=0, k=None, v=None, table=None), q=None, lens=None, o=None, ws=None, ws_bytes=0) == 0
    assert attend(lib, None) == 1


@pytest.mark.parametrize("change,status", [
    (dict(rows=-1), 1), (dict(vocab=0), 1), (dict(ld=99), 1), (dict(dtype=3), 1), (dict(dtype=-1), 1),
    (dict(logits=None), 1), (dict(u=None), 1), (dict(token=None), 1),
    (dict(vocab=262145, ld=262145), 2), (dict(rows=65536), 2),
    (dict(logits=1), 3), (dict(logits=2, dtype=2), 3), (dict(t=2), 3), (dict(k=2), 3), (dict(p=1), 3), (dict(m=3), 3),
    (dict(u=6), 3), (dict(token=2), 3), (dict(logprob=1), 3),
    (dict(rows=0, logits=None, u=None, token=None), 0),
])
def test_sample_validates_arguments(lib, change, status):
    a = dict(logits=2, dtype=0, ld=100, rows=2, vocab=100, t=None, k=None, p=None, m=None, u=4, token=4, logprob=None)
    a.update(change)
    assert lib.p4q_sample(a["logits"], a["dtype"], a["ld"], a["rows"], a["vocab"], a["t"], a["k"], a["p"], a["m"],
                          a["u"], a["token"], a["logprob"], None) == status


def test_status_of_a_bad_index_has_a_name(lib):
    lib.p4q_status_string.restype = ctypes.c_char_p
    lib.p4q_status_string.argtypes = [I]
    assert b"index" in lib.p4q_status_string(8)


def test_no_device_is_reported(lib):
    import torch
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    assert append(lib, paged()) == 7
    assert attend(lib, paged()) == 7
    assert lib.p4q_sample(2, 0, 100, 2, 100, None, None, None, None, 4, 4, None, None) == 7


def test_the_binding_refuses_what_it_cannot_pass():
    """Types and shapes that the C interface cannot see (the tensors lie on the CPU)."""
    import torch

    from paper_2609_34867_gb300 import p4q
    q = torch.zeros((2, 1024), dtype=torch.float16)
    cache = torch.zeros((16, 16, 4, 128), dtype=torch.float16)
    table = torch.zeros((2, 8), dtype=torch.int32)
    with pytest.raises(TypeError):
        p4q._paged_kv(cache, cache, table)  # not on a GPU
    with pytest.raises(TypeError):
        p4q.p4q_paged_attention(q, cache, cache, table, table[:, 0], q, None)
    with pytest.raises(TypeError):
        p4q.p4q_sample(q, torch.zeros(2), torch.zeros(2, dtype=torch.int32))
