"""Host-side checks of the entry points of a cache of codes (no GPU needed): what is
refused is refused before anything is launched."""
import ctypes

import pytest

from paper_2609_34867_gb300 import build as B

P, I, S = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
I64, I32 = ctypes.c_int64, ctypes.c_int32


class Codes(ctypes.Structure):
    _fields_ = [("k", P), ("v", P), ("k_scale", P), ("v_scale", P), ("table", P), ("page_stride", I64),
                ("token_stride", I64), ("head_stride", I64), ("scale_page_stride", I64), ("scale_token_stride", I64),
                ("scale_head_stride", I64), ("bits", I32), ("pages", I32), ("page_size", I32), ("Hkv", I32),
                ("dh", I32), ("seqs", I32), ("table_ld", I32), ("table_cols", I32)]


@pytest.fixture(scope="module")
def lib():
    B.build()
    L = ctypes.CDLL(B.LIB)
    L.p4q_rope_append_quant.argtypes = [P, I, P, I, P, I, I, I, P, P, I, I, I, P, P, P, ctypes.POINTER(Codes), I, P, I, P,
                                        I, P, I, P]
    L.p4q_paged_attention_quant.argtypes = [P, I, I, ctypes.POINTER(Codes), I, P, ctypes.c_float, P, I, P, P, S, P]
    L.p4q_paged_attention_workspace_bytes.argtypes = []
    L.p4q_paged_attention_workspace_bytes.restype = S
    return L


def codes(**changes):
    """A cache of 16 pages of 16 slots, 4 heads of 128 bytes, two sequences of 8 pages."""
    v = dict(k=16, v=16, k_scale=4, v_scale=4, table=4, page_stride=16 * 4 * 128, token_stride=4 * 128, head_stride=128,
             scale_page_stride=64, scale_token_stride=1, scale_head_stride=16, bits=8, pages=16, page_size=16, Hkv=4,
             dh=128, seqs=2, table_ld=8, table_cols=8)
    v.update(changes)
    return Codes(**v)


BAD_CACHES = [
    (dict(k=None), 1), (dict(v=None), 1), (dict(k_scale=None), 1), (dict(v_scale=None), 1), (dict(table=None), 1),
    (dict(pages=-1), 1), (dict(page_size=0), 1), (dict(Hkv=0), 1), (dict(dh=0), 1), (dict(seqs=-1), 1),
    (dict(table_ld=7), 1), (dict(table_cols=-1, table_ld=0), 1), (dict(page_stride=0), 1), (dict(token_stride=64), 1),
    (dict(head_stride=-128), 1), (dict(bits=4, head_stride=48), 1), (dict(scale_page_stride=0), 1),
    (dict(scale_token_stride=-1), 1), (dict(scale_head_stride=0), 1),
    (dict(bits=2), 2), (dict(bits=16), 2), (dict(page_size=24), 2), (dict(page_size=1 << 17), 2), (dict(dh=96), 2),
    (dict(Hkv=65536), 2),
    (dict(page_stride=8200), 3), (dict(token_stride=520), 3), (dict(head_stride=136), 3), (dict(k=8), 3),
    (dict(v=24), 3), (dict(k_scale=2), 3), (dict(v_scale=6), 3), (dict(table=2), 3),
]


def append(lib, kv, q=16, ldq=1024, k=16, ldk=512, v=16, ldv=512, T=2, H=8, cos=16, sin=16, max_pos=64, rot=128,
           inter=0, pos=4, rot_pos=None, seq=None, dtype=0, q_out=16, ldqo=1024, k_out=None, ldko=0, v_out=None, ldvo=0):
    return lib.p4q_rope_append_quant(q, ldq, k, ldk, v, ldv, T, H, cos, sin, max_pos, rot, inter, pos, rot_pos, seq,
                                     ctypes.byref(kv) if kv is not None else None, dtype, q_out, ldqo, k_out, ldko,
                                     v_out, ldvo, None)


def attend(lib, kv, q=16, ldq=1024, H=8, dtype=0, lens=4, scale=0.1, o=16, ldo=1024, lse=None, ws=16, ws_bytes=1 << 30):
    return lib.p4q_paged_attention_quant(q, ldq, H, ctypes.byref(kv) if kv is not None else None, dtype, lens, scale, o,
                                         ldo, lse, ws, ws_bytes, None)


@pytest.mark.parametrize("change,status", BAD_CACHES)
def test_cache_descriptions_are_checked(lib, change, status):
    assert append(lib, codes(**change)) == status
    assert attend(lib, codes(**change)) == status


@pytest.mark.parametrize("change,status", [
    (dict(T=-1), 1), (dict(H=0), 1), (dict(max_pos=0), 1), (dict(rot=0), 1), (dict(ldq=1016), 1), (dict(ldk=504), 1),
    (dict(ldv=504), 1), (dict(ldqo=512), 1), (dict(k_out=16, ldko=256), 1), (dict(v_out=16, ldvo=256), 1),
    (dict(q=None), 1), (dict(k=None), 1), (dict(v=None), 1), (dict(cos=None), 1), (dict(sin=None), 1),
    (dict(pos=None), 1), (dict(q_out=None), 1), (dict(T=3), 1),  # more tokens than sequences, and no seq
    (dict(rot=24), 2), (dict(rot=144), 2), (dict(H=65536, ldq=1 << 24, ldqo=1 << 24), 2), (dict(dtype=2), 2),
    (dict(dtype=-1), 2), (dict(ldq=1028), 3), (dict(ldk=516), 3), (dict(ldv=516), 3), (dict(ldqo=1028), 3),
    (dict(k_out=16, ldko=516), 3), (dict(v_out=16, ldvo=516), 3), (dict(q=8), 3), (dict(k=8), 3), (dict(v=8), 3),
    (dict(cos=8), 3), (dict(sin=4), 3), (dict(q_out=2), 3), (dict(k_out=8, ldko=512), 3), (dict(v_out=8, ldvo=512), 3),
    (dict(pos=2), 3), (dict(rot_pos=1), 3), (dict(seq=6), 3),
])
def test_append_validates_arguments(lib, change, status):
    assert append(lib, codes(), **change) == status


@pytest.mark.parametrize("change,status", [
    (dict(H=0), 1), (dict(H=6), 1), (dict(scale=float("nan")), 1), (dict(scale=float("inf")), 1), (dict(scale=3e38), 1),
    (dict(ldq=512), 1), (dict(ldo=512), 1), (dict(q=None), 1), (dict(lens=None), 1), (dict(o=None), 1),
    (dict(H=65536, ldq=1 << 24, ldo=1 << 24), 2), (dict(dtype=2), 2), (dict(ldq=1028), 3), (dict(ldo=1028), 3),
    (dict(q=8), 3), (dict(o=24), 3), (dict(lens=2), 3), (dict(lse=2), 3), (dict(ws=None), 4), (dict(ws_bytes=64), 4),
    (dict(ws=8), 3),
])
def test_attention_validates_arguments(lib, change, status):
    assert attend(lib, codes(), **change) == status


def test_missing_descriptions_and_empty_calls(lib):
    assert append(lib, None) == 1 and attend(lib, None) == 1
    none = codes(k=None, v=None, k_scale=None, v_scale=None, table=None, seqs=0)
    assert append(lib, none, T=0, q=None, k=None, v=None, cos=None, sin=None, pos=None, q_out=None) == 0
    assert attend(lib, none, q=None, lens=None, o=None, ws=None, ws_bytes=0) == 0
