"""Attention behind shared prefixes where the scores are so large that half a place of theirs is more
than the weights' exponents have room for. The values are fp16 or bf16 and finite; one
position of a head outweighs all others, so the output is that position's value.

Which position it is follows in 64 bits; only heads whose largest score is ahead of the second by more than
2 d + 64 are looked at, d = 2^-23 (dh A + 2 S + 8) the error of a score in fp32 (A the largest sum
|q_d k_d| scale, S the largest |score|): then the others' weights are below 2^-64 each, however the scores are
rounded. What is left of the bound of the other tests is u |o| + 2 (a + 2^-19) vmax + 2^-25, and d + a +
2^-22 |lse| for the logarithm of the sum."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DT = {"fp16": (torch.float16, 2.0 ** -11), "bf16": (torch.bfloat16, 2.0 ** -8)}


def make(dev, dt, dh, H, Hkv, n, prefix, own, size, seed, page=16):
    g = torch.Generator(device=dev).manual_seed(seed)
    dtype = DT[dt][0]
    length = prefix + own
    per = (length + page - 1) // page
    table = torch.arange(n * per, dtype=torch.int32, device=dev).view(n, per)
    table[:, :prefix // page] = table[0, :prefix // page]
    # up to 60000: fp16 ends at 65504
    large = lambda *shape: (torch.randn(shape, generator=g, device=dev) * size).clamp(-60000, 60000).to(dtype)  # noqa: E731
    k, q = large(n * per, page, Hkv, dh), large(n, H * dh)
    v = torch.randn((n * per, page, Hkv, dh), generator=g, device=dev).to(dtype)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)  # noqa: E731
    return q, k, v, table, i32([length] * n), i32([0, n]), i32([prefix])


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("size", [3000.0, 10000.0, 30000.0])
@pytest.mark.parametrize("n,H,Hkv,prefix,own,scale", [
    (6, 16, 4, 400, 30, None),       # four copies of a tile's rows
    (12, 32, 8, 700, 200, None),     # two
    (40, 24, 2, 1000, 3, None),      # one, several tiles
    (9, 8, 2, 300, 40, -0.1)])
def test_one_position_outweighs_the_others(p4q, dev, dt, dh, size, n, H, Hkv, prefix, own, scale):
    q, k, v, table, lens, start, shared = make(dev, dt, dh, H, Hkv, n, prefix, own, size, seed=n + dh)
    ws = p4q.prefix_attention_workspace(n, 1, H, dh, dev)
    o, lse = torch.empty_like(q), torch.empty((n, H), device=dev)
    p4q.p4q_prefix_attention(q, k, v, table, lens, start, shared, o, ws, scale=scale, lse=lse)
    torch.cuda.synchronize()
    assert p4q.p4q_device_status() == 0
    scale = dh ** -0.5 if scale is None else scale
    seen, u = 0, DT[dt][1]
    for b in range(n):
        length = prefix + own
        kb, vb = (torch.cat((x[table[0].long()].flatten(0, 1)[:prefix], x[table[b].long()].flatten(0, 1)[prefix:length])).double()
                  for x in (k, v))
        qb = q[b].double().view(Hkv, H // Hkv, dh)
        s = (torch.einsum("hgd,lhd->hgl", qb, kb) * scale).reshape(H, length)
        A = (torch.einsum("hgd,lhd->hgl", qb.abs(), kb.abs()) * abs(scale)).amax(-1).reshape(H)
        S = s.abs().amax(-1)
        d = 2.0 ** -23 * (dh * A + 2 * S + 8)
        top, which = s.topk(2, -1)
        clear = top[:, 0] - top[:, 1] > 2 * d + 64
        seen += int(clear.sum())
        vh = vb.permute(1, 0, 2).repeat_interleave(H // Hkv, 0)  # [H, length, dh]
        want = vh[torch.arange(H, device=dev), which[:, 0]]
        vmax = vh.abs().amax((1, 2))
        a = 2.0 ** -24 * (64 + length / 16)
        got, glse = o[b].double().view(H, dh), lse[b].double()
        bound = u * want.abs() + 2 * (a + 2.0 ** -19) * vmax[:, None] + 2.0 ** -25
        assert bool(((got - want).abs() <= bound)[clear].all()), f"sequence {b}"
        assert bool(((glse - top[:, 0]).abs() <= d + a + 2.0 ** -22 * top[:, 0].abs())[clear].all()), f"sequence {b}"
    assert seen >= n * H // 2, "too few heads have one position ahead"
