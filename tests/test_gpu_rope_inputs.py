"""The rotary append leaves its inputs as they are where it does not rotate in place,
and everything beside the rows that it writes."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("inter,rot,dh", [(False, 128, 128), (True, 64, 128), (False, 32, 64)])
@pytest.mark.parametrize("T", [1, 3, 130])
@pytest.mark.parametrize("in_place", [False, True])
def test_what_is_not_written_stays(p4q, dev, dt, inter, rot, dh, T, in_place):
    H, Hkv, page, pad, gap = 6, 2, 16, 8, 16
    g = torch.Generator(device=dev).manual_seed(T)
    rand = lambda *s: torch.randn(s, generator=g, device=dev).to(dt)  # noqa: E731
    # q, k and v as column blocks of one row, with columns of nobody behind each
    fused = rand(T, (H + 2 * Hkv) * dh + 3 * gap)
    at = {}
    c = 0
    for name, heads in (("q", H), ("k", Hkv), ("v", Hkv)):
        at[name] = (c, c + heads * dh)
        c += heads * dh + gap
    q, k, v = (fused[:, a:b] for a, b in at.values())
    out = rand(T, (H + Hkv) * dh + 2 * pad)
    q_out, k_out = (q, k) if in_place else (out[:, :H * dh], out[:, H * dh + pad:(H + Hkv) * dh + pad])
    pages = (T + page - 1) // page + 2
    cache = [rand(pages, page, Hkv, dh) for _ in range(2)]
    table = torch.randperm(pages, generator=g, device=dev).to(torch.int32)[None]
    pos, seq = torch.arange(T, dtype=torch.int32, device=dev), torch.zeros(T, dtype=torch.int32, device=dev)
    ang = torch.rand((T, rot // 2), generator=g, device=dev) * 6
    cos, sin = ang.cos(), ang.sin()
    given = [t.clone() for t in (fused, out, *cache, table, pos, seq, cos, sin)]
    p4q.p4q_rope_append(q, k, v, cos, sin, pos, *cache, table, q_out, k_out=k_out, seq=seq, interleaved=inter)
    torch.cuda.synchronize()
    assert p4q.p4q_device_status() == 0
    fused0, out0, k0, v0 = given[:4]
    for now, then in zip((table, pos, seq, cos, sin), given[4:]):
        assert torch.equal(now, then)
    assert torch.equal(v, fused0[:, slice(*at["v"])])
    if in_place:
        assert torch.equal(out, out0)
        mine = torch.zeros(fused.shape[1], dtype=torch.bool, device=dev)
        for name in ("q", "k"):
            mine[slice(*at[name])] = True
        assert torch.equal(fused[:, ~mine], fused0[:, ~mine])
    else:
        assert torch.equal(fused, fused0)
        mine = torch.ones(out.shape[1], dtype=torch.bool, device=dev)
        mine[H * dh:H * dh + pad] = False
        mine[-pad:] = False
        assert torch.equal(out[:, ~mine], out0[:, ~mine])
    # the cache: only the tokens' slots
    named = torch.zeros((pages, page), dtype=torch.bool, device=dev)
    named[table[0, torch.arange(T, device=dev) // page].long(), torch.arange(T, device=dev) % page] = True
    for now, then in zip(cache, (k0, v0)):
        assert torch.equal(now[~named], then[~named])
    assert torch.equal(cache[1][table[0, pos.long() // page].long(), pos.long() % page].reshape(T, -1), v)
