"""The allocating wrappers of attention over codes and of shared prefixes on another stream than the current
one: what they allocate is not memory that was freed on the current stream, and the results are the same.
Refusals of the Python binding: a wrong argument is named, whatever else is right."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _cases(p4q, dev):
    g = torch.Generator(device=dev).manual_seed(3)
    half = lambda *s: torch.randn(s, generator=g, device=dev).half()  # noqa: E731
    table = torch.arange(20, dtype=torch.int32, device=dev).view(2, 10)
    lens = torch.tensor([150, 77], dtype=torch.int32, device=dev)
    q = half(2, 512)
    codes = [torch.randint(-127, 128, (20, 16, 2, 128), generator=g, device=dev, dtype=torch.int8) for _ in range(2)]
    scales = [torch.rand((20, 16, 2), generator=g, device=dev) for _ in range(2)]
    cache = [half(20, 16, 2, 128) for _ in range(2)]
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=dev)  # noqa: E731
    return {"paged_attention_quant": lambda **k: p4q.paged_attention_quant(q, *codes, *scales, table, lens, **k),
            "prefix_attention": lambda **k: p4q.prefix_attention(q, *cache, table, lens, i32(0, 2), i32(64), **k)}


@pytest.mark.parametrize("name", ["paged_attention_quant", "prefix_attention"])
def test_another_stream(p4q, dev, name):
    call = _cases(p4q, dev)[name]
    want = call().clone()
    torch.cuda.synchronize()
    old = torch.empty_like(want)
    at = old.data_ptr()
    del old
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = call(stream=s)
    assert got.data_ptr() != at
    s.synchronize()
    assert torch.equal(got, want)


def test_wrong_arguments_are_named(p4q, dev):
    g = torch.Generator(device=dev).manual_seed(3)
    n, H, Hkv, dh, page = 2, 4, 2, 128, 16
    codes = [torch.zeros((8, page, Hkv, dh), dtype=torch.int8, device=dev) for _ in range(2)]
    scales = [torch.zeros((8, page, Hkv), device=dev) for _ in range(2)]
    cache = [torch.zeros((8, page, Hkv, dh), dtype=torch.float16, device=dev) for _ in range(2)]
    table = torch.zeros((n, 4), dtype=torch.int32, device=dev)
    lens = torch.ones((n,), dtype=torch.int32, device=dev)
    q = torch.randn((n, H * dh), generator=g, device=dev).half()
    k = torch.zeros((n, Hkv * dh), dtype=torch.float16, device=dev)
    cos = torch.ones((4, 64), device=dev)
    o, ws = torch.empty_like(q), p4q.paged_attention_workspace(dev)
    pws = p4q.prefix_attention_workspace(n, 1, H, dh, dev)
    start, prefix = torch.tensor([0, 2], dtype=torch.int32, device=dev), torch.ones((1,), dtype=torch.int32, device=dev)

    def append(**c):
        a = dict(q=q, k=k, v=k.clone(), cos=cos, sin=cos, pos=lens, k_cache=codes[0], v_cache=codes[1], k_scale=scales[0],
                 v_scale=scales[1], table=table, q_out=o)
        a.update(c)
        p4q.p4q_rope_append_quant(**a)

    def attend(**c):
        a = dict(q=q, k_cache=codes[0], v_cache=codes[1], k_scale=scales[0], v_scale=scales[1], table=table, lens=lens, o=o, ws=ws)
        a.update(c)
        p4q.p4q_paged_attention_quant(**a)

    def share(**c):
        a = dict(q=q, k_cache=cache[0], v_cache=cache[1], table=table, lens=lens, group_start=start, prefix_lens=prefix, o=o, ws=pws)
        a.update(c)
        p4q.p4q_prefix_attention(**a)

    for call in (append, attend, share):
        call()
    before = p4q.p4q_launch_count()
    f32, i64 = q.float(), lens.long()
    for call, change, kind, what in (
            (append, dict(q=f32), TypeError, "q"), (append, dict(k=f32), TypeError, "k"), (append, dict(v=k[:1]), ValueError, "v"),
            (append, dict(pos=i64), TypeError, "pos"), (append, dict(k_cache=cache[0]), TypeError, "k_cache"),
            (append, dict(v_cache=codes[1][:4]), TypeError, "v_cache"), (append, dict(k_scale=scales[0].half()), TypeError, "k_scale"),
            (append, dict(v_scale=scales[1][:, :4]), TypeError, "v_scale"), (append, dict(table=table.long()), TypeError, "table"),
            (append, dict(cos=cos.half()), TypeError, "cos"), (append, dict(sin=cos[:2]), ValueError, "sin"),
            (append, dict(k_out=k[:, :128]), ValueError, "k_out"), (append, dict(v_out=f32), TypeError, "v_out"),
            (append, dict(seq=i64), TypeError, "seq"), (append, dict(q=q.cpu()), TypeError, "q"),
            (attend, dict(q=q[:1]), ValueError, "q"), (attend, dict(o=o[:, :256]), ValueError, "o"),
            (attend, dict(lens=lens[:1]), ValueError, "lens"), (attend, dict(ws=f32), TypeError, "ws"),
            (attend, dict(lse=torch.empty((n, 3), device=dev)), ValueError, "lse"), (attend, dict(k_cache=None), TypeError, "k_cache"),
            (share, dict(k_cache=codes[0]), TypeError, "k_cache"), (share, dict(prefix_lens=None), TypeError, "prefix_lens"),
            (share, dict(group_start=start[:1]), ValueError, "group_start"), (share, dict(lens=i64), TypeError, "lens"),
            (share, dict(q=q.bfloat16()), TypeError, "q")):
        with pytest.raises(kind, match=what):
            call(**change)
    for call, change in ((attend, dict(ws=ws[:64])), (share, dict(ws=pws[:-32])), (attend, dict(scale=float("nan"))),
                         (append, dict(q_out=o.view(-1)[4:4 + 1020].as_strided((2, 512), (508, 1))))):
        with pytest.raises(p4q.P4QError):
            call(**change)
    assert p4q.p4q_launch_count() == before
    torch.cuda.synchronize()
    assert p4q.p4q_device_status() == 0
