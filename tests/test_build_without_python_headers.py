"""The library's build where Python has no headers: libp4q.so is built all the same, and the binding
marshals the calls of a decode step by itself."""
import os
import sysconfig

import pytest
import torch

from paper_2609_34867_gb300 import build as B, p4q


@pytest.fixture
def small(tmp_path, monkeypatch):
    """The build with one small source, into a folder of its own."""
    src = tmp_path / "one.cu"
    src.write_text('extern "C" int p4q_one() { return 1; }\n')
    for name, value in (("LIBDIR", tmp_path), ("LIB", tmp_path / "libp4q.so"), ("CALL", tmp_path / "p4q_call.so")):
        monkeypatch.setattr(B, name, str(value))
    monkeypatch.setattr(B, "sources", lambda: [str(src)])
    return tmp_path


def without_headers(monkeypatch, folder):
    paths = dict(sysconfig.get_paths(), include=str(folder))
    monkeypatch.setattr(sysconfig, "get_paths", lambda *a, **k: paths)


def test_the_library_is_built_without_headers(small, monkeypatch):
    without_headers(monkeypatch, small)
    (small / "p4q_call.so").write_bytes(b"of another source")
    B.build()
    assert os.path.exists(B.LIB) and not os.path.exists(B.CALL) and not list(small.glob("*.tmp*"))
    built = os.path.getmtime(B.LIB)
    assert B.up_to_date()
    B.build()
    assert os.path.getmtime(B.LIB) == built


@pytest.mark.skipif(B.python_headers() is None, reason="Python has no headers here")
def test_the_module_is_built_with_headers(small):
    B.build()
    assert os.path.exists(B.LIB) and os.path.exists(B.CALL) and B.up_to_date()


@pytest.mark.skipif(B.python_headers() is None, reason="Python has no headers here")
def test_a_module_that_fails_is_named_and_leaves_the_library(small, monkeypatch):
    bad = small / "csrc"
    bad.mkdir()
    (bad / "p4q_call.c").write_text("not C\n")
    monkeypatch.setattr(B, "CSRC", str(bad))
    with pytest.raises(RuntimeError, match="p4q_call.c"):
        B.build()
    assert os.path.exists(B.LIB)


def test_arguments_are_refused_without_the_module(monkeypatch, tmp_path):
    B.build()
    monkeypatch.setattr(B, "CALL", str(tmp_path / "none.so"))
    monkeypatch.setattr(p4q, "_fast", None)
    cache = [torch.zeros((2, 16, 1, 128), dtype=torch.int8)] * 2 + [torch.zeros((2, 16, 1))] * 2
    q, table, lens = torch.zeros((1, 128)).half(), torch.zeros((1, 2), dtype=torch.int32), torch.ones((1,), dtype=torch.int32)
    with pytest.raises(TypeError, match="k_cache"):  # not on a GPU
        p4q.p4q_paged_attention_quant(q, *cache, table, lens, q, lens)
    with pytest.raises(TypeError, match="k_cache"):
        p4q.p4q_prefix_attention(q, cache[0].half(), cache[0].half(), table, lens, lens, lens, q, lens)
    with pytest.raises(TypeError, match="k_cache"):
        p4q.p4q_rope_append_quant(q, q, q, q, q, lens, *cache, table, q)
    assert p4q._fast is p4q._NoCall


@pytest.mark.gpu
def test_the_calls_give_the_same_without_the_module(monkeypatch, tmp_path, dev):
    B.build()
    g = torch.Generator(device=dev).manual_seed(1)
    rnd = lambda *s: torch.randn(s, generator=g, device=dev).half()  # noqa: E731
    n, H, Hkv, dh, page, per = 5, 8, 2, 128, 16, 4
    q, k, v = rnd(n, H * dh), rnd(n, Hkv * dh), rnd(n, Hkv * dh)
    table = torch.randperm(n * per, generator=g, device=dev).to(torch.int32).view(n, per)
    table[:, :2] = table[0, :2]
    lens = torch.tensor([40, 64, 33, 50, 41], dtype=torch.int32, device=dev)
    cos, sin = torch.rand((64, 64), generator=g, device=dev), torch.rand((64, 64), generator=g, device=dev)
    kc, vc = rnd(n * per, page, Hkv, dh), rnd(n * per, page, Hkv, dh)
    start, prefix = torch.tensor([0, n], dtype=torch.int32, device=dev), torch.tensor([32], dtype=torch.int32, device=dev)

    def calls():
        codes = [torch.zeros((n * per, page, Hkv, dh), dtype=torch.int8, device=dev) for _ in range(2)]
        scales = [torch.zeros((n * per, page, Hkv), device=dev) for _ in range(2)]
        qo, ko, lse = torch.empty_like(q), torch.empty_like(k), torch.empty((n, H), device=dev)
        p4q.p4q_rope_append_quant(q, k, v, cos, sin, lens - 1, *codes, *scales, table, qo, k_out=ko)
        o = p4q.paged_attention_quant(qo, *codes, *scales, table, lens, scale=0.1)
        o2 = torch.empty_like(q)
        p4q.p4q_prefix_attention(q, kc, vc, table, lens, start, prefix, o2, p4q.prefix_attention_workspace(n, 1, H, dh, dev),
                                 lse=lse)
        torch.cuda.synchronize()
        return [*codes, *scales, qo, ko, o, o2, lse]

    with_module = calls()
    monkeypatch.setattr(B, "CALL", str(tmp_path / "none.so"))
    monkeypatch.setattr(p4q, "_fast", None)
    without = calls()
    assert p4q._fast is p4q._NoCall
    assert all(torch.equal(a, b) for a, b in zip(with_module, without))
    assert p4q.p4q_device_status() == 0
