"""Attention over a cache of codes whose values' scales fall while the scores rise, so that what
counts at the end of a sequence is far below the largest scale before it. Against the formula in 64 bits.

q and the keys have one dimension that is not 0, so the scores have the three roundings of their factors
and difference: d = 2^-23 (4 S + 8), S the largest |score|. M is the sum of weights times scales times 127 or 7 (not
the largest value of the head, whatever its weight): weights times scales enter as two fp16 values, 2^-21 of each and
2^-34 of the largest one so far for each of up to 2^12 positions, 2^-19 M at most. Bound: u |o| + 2 (d + a + 2^-19) M
(+ 2^-25 for an fp16 output), a = 2^-24 (64 + n / 16) from adding n weights in parts."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

DT = {"fp16": (torch.float16, 2.0 ** -11, 2.0 ** -25), "bf16": (torch.bfloat16, 2.0 ** -8, 2.0 ** -134)}


def pack(c):
    return ((c[..., 0::2] & 15) | (c[..., 1::2] << 4)).view(torch.uint8)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("dh,page", [(128, 16), (64, 8), (64, 64)])
@pytest.mark.parametrize("form,fall", [("jump", 24), ("jump", 30), ("jump", 40), ("jump", 90), ("stairs", 8), ("stairs", 3), ("there and back", 40)])
@pytest.mark.parametrize("n,Hkv,length", [(80, 8, 2048), (2, 2, 1500)])
def test_what_counts_is_far_below_an_earlier_scale(p4q, dev, bits, dt, dh, page, form, fall, n, Hkv, length):
    g = torch.Generator(device=dev).manual_seed(fall)
    dtype, u, least = DT[dt]
    H, most, per = 4 * Hkv, 127 if bits == 8 else 7, (length + page - 1) // page
    j = torch.arange(per * page, device=dev)
    if form == "jump":  # the second half: scores higher by `fall` + 2 powers of two, scales lower by `fall`
        power = torch.where(j < length // 2, float(fall), 0.0)
        rise = torch.where(j < length // 2, 0.0, fall + 2.0)
    elif form == "stairs":  # by `fall` and a little more than a reference lets pass, every 256 positions
        steps = j // 256
        power, rise = (per * page // 256 - steps) * float(fall), steps * (fall + 1.5 if fall == 8 else 9.5)
    else:  # large scales of no weight at the end again
        third = j * 3 // length
        power = torch.where(third == 1, 0.0, float(fall))
        rise = torch.where(third == 1, fall + 2.0, 0.0)
    jitter = torch.rand((n * per, page, Hkv), generator=g, device=dev)
    ks = ((rise.view(1, per, page, 1) * math.log(2)).expand(n, -1, -1, Hkv).reshape(n * per, page, Hkv) + jitter).contiguous()
    vs = ((2.0 ** power).view(1, per, page, 1).expand(n, -1, -1, Hkv).reshape(n * per, page, Hkv)
          * (1 + torch.rand((n * per, page, Hkv), generator=g, device=dev)) / most).contiguous()
    kc = torch.zeros((n * per, page, Hkv, dh), dtype=torch.int8, device=dev)
    kc[..., 0] = 1
    vc = torch.randint(-most, most + 1, (n * per, page, Hkv, dh), generator=g, device=dev, dtype=torch.int8)
    q = torch.zeros((n, H, dh), device=dev)
    q[..., 0] = 1 + torch.randint(0, 3, (n, H), generator=g, device=dev) / 64.0
    q = q.to(dtype).view(n, H * dh)
    table = torch.randperm(n * per, generator=g, device=dev).to(torch.int32).view(n, per)
    back = torch.argsort(table.reshape(-1).long())  # page table[b][i] is the i-th of sequence b
    cache = [x[back].contiguous() for x in ((kc, vc) if bits == 8 else (pack(kc), pack(vc)))]
    scales = [x[back].contiguous() for x in (ks, vs)]
    lens = torch.full((n,), length, dtype=torch.int32, device=dev)
    o, lse = torch.empty_like(q), torch.empty((n, H), device=dev)
    p4q.p4q_paged_attention_quant(q, *cache, *scales, table, lens, o, p4q.paged_attention_workspace(dev), scale=1.0, lse=lse)
    torch.cuda.synchronize()
    assert p4q.p4q_device_status() == 0
    for b in range(0, n, 13):
        at = slice(b * per, (b + 1) * per)
        k1, s1 = (x[at].flatten(0, 1)[:length].double() for x in (ks, vs))          # [length, Hkv]
        v = vc[at].flatten(0, 1)[:length].double() * s1[..., None]
        s = (q[b].double().view(Hkv, 4, dh)[..., 0][..., None] * k1.t()[:, None, :])  # [Hkv, 4, length]
        w = torch.softmax(s, -1)
        want = torch.einsum("hgl,lhd->hgd", w, v).reshape(H, dh)
        M = most * torch.einsum("hgl,lh->hg", w, s1).reshape(H, 1)
        d = 2.0 ** -23 * (4 * s.abs().amax(-1).reshape(H, 1) + 8)
        a = 2.0 ** -24 * (64 + length / 16)
        bound = u * want.abs() + 2 * (d + a + 2.0 ** -19) * M + least
        err = (o[b].double().view(H, dh) - want).abs()
        assert bool((err <= bound).all()), f"sequence {b}: {float((err / bound).max()):.3g} of the bound"
        wlse = torch.logsumexp(s, -1).reshape(H)
        assert bool(((lse[b].double() - wlse).abs() <= d[:, 0] + a + 2.0 ** -22 * wlse.abs()).all())
