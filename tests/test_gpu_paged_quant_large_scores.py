"""Attention over a cache of codes where the scores are so large that half a place of theirs is more
than the weights' exponents have room for; q is finite and below 2^118. One position of a
head outweighs all others, so the output is that position's value.

Which position it is follows in 64 bits; only heads whose largest score is ahead of the second by more than
2 d + 64 are looked at, d = 2^-23 (dh A + 4 S + 8) the error of a score (S the largest |score|, A the largest
sum |q_d m_d| scale, m_d = |k_d|, at 4 bits 15 scales of k: the keys' nibbles are counted from -8): then the
others' weights are below 2^-64 each, however the scores are rounded. What is left of the bound of the other
tests is u |o| + 2 (a + 2^-19) vmax + 2^-25, and d + a + 2^-22 |lse| for the logarithm of the sum."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DT = {"fp16": (torch.float16, 2.0 ** -11), "bf16": (torch.bfloat16, 2.0 ** -8)}


def pack(c):
    return ((c[..., 0::2] & 15) | (c[..., 1::2] << 4)).view(torch.uint8)


def make(dev, bits, dt, dh, H, Hkv, n, length, size, key_scale, seed, page=16):
    g = torch.Generator(device=dev).manual_seed(seed)
    per, most = (length + page - 1) // page, 127 if bits == 8 else 7
    table = torch.arange(n * per, dtype=torch.int32, device=dev).view(n, per)
    codes = [torch.randint(-most, most + 1, (n * per, page, Hkv, dh), generator=g, device=dev, dtype=torch.int8) for _ in range(2)]
    ks, vs = ((torch.rand((n * per, page, Hkv), generator=g, device=dev) + 0.5) * f / most for f in (key_scale, 1.0))
    q = torch.randn((n, H * dh), generator=g, device=dev) * size
    q = (q.clamp(-60000, 60000) if dt == "fp16" else q).to(DT[dt][0])
    return q, codes, ks, vs, table


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("dt,size,key_scale", [("fp16", 30000.0, 1e3), ("fp16", 30000.0, 1e8), ("fp16", 1.0, 1e14), ("bf16", 1e6, 1.0),
                                               ("bf16", 1e9, 1.0), ("bf16", 1e13, 1.0), ("bf16", 1e30, 1e-3)])
@pytest.mark.parametrize("n,H,Hkv,length,scale", [(3, 16, 4, 430, None), (70, 32, 8, 900, None), (6, 24, 2, 700, -0.1),
                                                  (2, 8, 8, 64, None)])
def test_one_position_outweighs_the_others(p4q, dev, bits, dt, dh, size, key_scale, n, H, Hkv, length, scale):
    q, (kc, vc), ks, vs, table = make(dev, bits, dt, dh, H, Hkv, n, length, size, key_scale, seed=n + dh)
    o, lse = torch.empty_like(q), torch.empty((n, H), device=dev)
    lens = torch.full((n,), length, dtype=torch.int32, device=dev)
    cache = (kc, vc) if bits == 8 else (pack(kc), pack(vc))
    p4q.p4q_paged_attention_quant(q, *cache, ks, vs, table, lens, o, p4q.paged_attention_workspace(dev), scale=scale, lse=lse)
    torch.cuda.synchronize()
    assert p4q.p4q_device_status() == 0
    scale = dh ** -0.5 if scale is None else scale
    seen, u = 0, DT[dt][1]
    for b in range(0, n, 7):
        at = table[b].long()
        kb, vb = ((c[at].double() * s[at].double()[..., None]).flatten(0, 1)[:length] for c, s in ((kc, ks), (vc, vs)))
        mags = kb.abs() if bits == 8 else (15 * ks[at].double()).flatten(0, 1)[:length, :, None].expand(-1, -1, dh)
        qb = q[b].double().view(Hkv, H // Hkv, dh)
        s = (torch.einsum("hgd,lhd->hgl", qb, kb) * scale).reshape(H, length)
        A = (torch.einsum("hgd,lhd->hgl", qb.abs(), mags) * abs(scale)).amax(-1).reshape(H)
        d = 2.0 ** -23 * (dh * A + 4 * s.abs().amax(-1) + 8)
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
    assert seen >= len(range(0, n, 7)) * H // 2, "too few heads have one position ahead"
