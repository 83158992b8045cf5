"""The allocating wrappers on another stream than the current one: what they allocate
is not memory that was freed on the current stream, where work on it may be under way,
and a workspace that a wrapper drops is not handed to the current stream while its
kernels may still write it."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _cases(p4q, dev):
    g = torch.Generator(device=dev).manual_seed(3)
    half = lambda *s: torch.randn(s, generator=g, device=dev).half()  # noqa: E731
    X, W = half(40, 512), half(256, 512)
    Xq, sa = p4q.quant_act(X)
    Wq, sw = p4q.quant_weight(W)
    V, Q, A, text = half(2, 200, 256), half(2, 3, 256), torch.rand((2, 200), generator=g, device=dev), half(2, 5, 256)
    cache = [half(20, 16, 2, 128) for _ in range(2)]
    table = torch.arange(20, dtype=torch.int32, device=dev).view(2, 10)
    lens = torch.tensor([150, 77], dtype=torch.int32, device=dev)
    q, u = half(2, 512), torch.rand((40,), generator=g, device=dev)
    qc, kc, kp = half(2, 4, 4, 64), half(2, 4, 4, 64), half(2, 100, 4, 64)
    lin_ws = p4q.linear_workspace(40, 256, 512, dev)
    return {
        "quant_act": lambda **k: p4q.quant_act(X, **k),
        "quant_weight": lambda **k: p4q.quant_weight(W, **k),
        "w4a4_linear": lambda **k: p4q.w4a4_linear(Xq, sa, Wq, sw, **k),
        "w4a4_gemm_s32": lambda **k: p4q.w4a4_gemm_s32(Xq, Wq, **k),
        "w4a4_gemm_s32_ws": lambda **k: p4q.w4a4_gemm_s32_ws(Xq, Wq, lin_ws, **k),
        "expand_codes": lambda **k: p4q.expand_codes(Xq, **k),
        "cls_saliency": lambda **k: p4q.cls_saliency(qc, kc, kp, **k),
        "select": lambda **k: p4q.select(V, Q, A, 64, **k),
        "select_gather_quant": lambda **k: p4q.select_gather_quant(V, Q, A, text, 64, **k),
        "paged_attention": lambda **k: p4q.paged_attention(q, *cache, table, lens, **k),
        "sample": lambda **k: p4q.sample(X, u, **k),
    }


@pytest.mark.parametrize("name", ["quant_act", "quant_weight", "w4a4_linear", "w4a4_gemm_s32", "w4a4_gemm_s32_ws",
                                  "expand_codes", "cls_saliency", "select", "select_gather_quant", "paged_attention", "sample"])
def test_memory_of_another_stream(p4q, dev, monkeypatch, name):
    call = _cases(p4q, dev)[name]
    many = lambda r: r if isinstance(r, tuple) else (r,)  # noqa: E731
    want = [t.clone() for t in many(call())]
    workspaces = []
    for make in ("paged_attention_workspace", "select_workspace"):
        def kept(*a, _make=getattr(p4q, make)):
            ws = _make(*a)
            workspaces.append((ws.data_ptr(), ws.numel()))
            return ws
        monkeypatch.setattr(p4q, make, kept)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    # memory of the outputs' sizes, freed on the current stream
    old = [torch.empty_like(t) for t in want]
    freed = {t.data_ptr() for t in old}
    del old
    s = torch.cuda.Stream()
    got = many(call(stream=s))
    s.synchronize()
    assert p4q.p4q_device_status() == 0
    assert not freed & {t.data_ptr() for t in got}
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    if name in ("select", "select_gather_quant", "paged_attention"):
        (at, size), = workspaces
        again = torch.empty((size,), dtype=torch.uint8, device=dev)  # on the current stream
        assert again.data_ptr() != at
    else:
        assert not workspaces
