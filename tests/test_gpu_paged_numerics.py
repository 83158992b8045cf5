"""What the paged attention's numbers hold beyond the general bounds: the softmax
weights keep the precision of fp32 in the product with the values, and infinite
values act as in the formula."""
import math

import pytest
import torch

from test_gpu_paged_attention import check, make, run

pytestmark = pytest.mark.gpu

TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}


def _rounded_twice(w, dtype):
    """w (fp64) as the sum of two values of dtype, each rounded to nearest."""
    hi = w.to(dtype).double()
    return hi + (w - hi).to(dtype).double()


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("page", [4, 16])
@pytest.mark.parametrize("H,Hkv,dh", [(2, 2, 128), (8, 1, 128), (12, 1, 128), (2, 1, 64), (16, 1, 64)])
def test_weights_keep_24_bits(p4q, dev, dt, page, H, Hkv, dh):
    """Scores are chosen so that their weights are the furthest from two values of
    bf16, half of them above and half below, and the values so that the sum is all but 0 in
    64 bits: what is left is the weights' error.

    Blocks of 16 positions begin with a score of 0, so that every warp's weights are the
    exponentials times a power of two. The scores are single products and exact. Error of a
    weight, relative: exponent's product and scale 3 * 2^-24 * 1.45, exponent's difference half a
    place of its range, both times ln 2, and the exponential 2^-22. The range is below 2 in bf16 (2^-24), below
    16 in fp16 (2^-21), whose weights are 2^11 times as large: below 2^-21 and 2^-20. Products with v
    are exact in fp32 (of p's parts); a sum of 17 addends in each of three products per block is
    off by 17 * 2^-23 of its largest partial sum, which is below 2 p v as signs alternate:
    four blocks, three products, divided by the weights' sum L (> 40): 408 * 2^-23 / L vmax.
    Output: rounded once, u |o| + 2^-25 for an fp16 value below its normal range. Weights of 16
    bits are off by 2^-18 and more, all in one direction."""
    dtype, u = TYPES[dt], {"fp16": 2.0 ** -11, "bf16": 2.0 ** -8}[dt]
    s = torch.arange(-256, -64, dtype=torch.float64) / 256  # -1 .. -1/4 in steps that bf16 and fp16 hold
    s = torch.cat((s, torch.arange(-127, -16, dtype=torch.float64) / 512))
    s = s[s == s.to(torch.bfloat16).double()]
    w = torch.exp(s)
    off = w - _rounded_twice(w, torch.bfloat16)
    order = torch.argsort(off)
    low, high = order[:30], order.flip(0)[:30]
    assert float(off[low].mean()) < -2.0 ** -20 and float(off[high].mean()) > 2.0 ** -20
    # by weight, so that neighbours of both signs all but cancel
    low, high = low[torch.argsort(w[low])], high[torch.argsort(w[high])]
    tested = torch.stack((high, low), 1).reshape(-1)
    score = torch.zeros((64,), dtype=torch.float64)
    value = torch.zeros((64,), dtype=torch.float64)
    at = torch.tensor([j for j in range(64) if j % 16])
    score[at] = s[tested]
    value[at] = torch.tensor([1.0, -1.0], dtype=torch.float64).repeat(30)
    weight = torch.exp(score)
    for j in (0, 16, 32, 48):  # the rest of the sum, rounded and again what is left
        value[j] = (-(weight * value).sum()).to(dtype).double()
    scale_v = (1.0 + torch.arange(dh, dtype=torch.float64) / 128)  # exact products of few bits
    scale_v = (scale_v * 8).round() / 8
    v = (value[:, None] * scale_v).to(dtype)
    k = torch.zeros((64, dh), dtype=dtype)
    k[:, 1:] = torch.randn((64, dh - 1), generator=torch.Generator().manual_seed(1)).to(dtype)
    k[:, 0] = score.to(dtype)
    assert torch.equal(k[:, 0].double(), score)
    pages = 64 // page
    table = torch.randperm(pages, generator=torch.Generator().manual_seed(2))
    kc, vc = (torch.zeros((pages, page, Hkv, dh), dtype=dtype) for _ in range(2))
    kc[table] = k.view(pages, page, 1, dh).expand(-1, -1, Hkv, -1)
    vc[table] = v.view(pages, page, 1, dh).expand(-1, -1, Hkv, -1)
    q = torch.zeros((1, H * dh), dtype=dtype)
    q[:, ::dh] = 1.0
    o = torch.empty((1, H * dh), dtype=dtype, device=dev)
    lse = torch.empty((1, H), device=dev)
    p4q.p4q_paged_attention(q.to(dev), kc.to(dev), vc.to(dev), table.to(torch.int32)[None].to(dev),
                            torch.tensor([64], dtype=torch.int32, device=dev), o, p4q.paged_attention_workspace(dev),
                            scale=1.0, lse=lse)
    torch.cuda.synchronize()
    assert p4q.p4q_device_status() == 0
    L = float(weight.sum())
    want = (weight[:, None] * v.double()).sum(0) / L
    vmax = v.double().abs().amax(0)
    size = (weight[:, None] * v.double().abs()).sum(0) / L
    d = {"fp16": 2.0 ** -20, "bf16": 2.0 ** -21}[dt]
    bound = u * want.abs() + (2.0 ** -25 if dt == "fp16" else 0.0) + d * size + 408 * 2.0 ** -23 / L * vmax
    err = (o.cpu().double().view(H, dh) - want).abs()
    assert bool((err <= bound).all()), f"largest {float((err / bound).max()):.2f} of the bound, {float(err.max()):.3g}"
    assert abs(float(lse.cpu().double()[0, 0]) - math.log(L)) <= 2.0 ** -20


def _non_finite(p4q, dev, lens, H, Hkv, dh, page, dt, put, qscale=1.0, seed=0):
    """Sequences with the values that put(b, v [len, Hkv, dh], g) writes among them, against
    the formula: dimensions that a non-finite value with a weight reaches are infinite or NaN as
    it says (infinite values whose weights are below 2^-100 of the largest are left out), the others have
    the finite sum, to the general bound."""
    c = make(dev, lens, H, Hkv, dh, page, dt, seed, qscale=qscale)
    g = torch.Generator(device=dev).manual_seed(seed + 1)
    for b, n in enumerate(lens):
        if n > 0:
            put(b, c["vs"][b], g)
            j = torch.arange(n, device=dev)
            c["v"][c["table"][b].long()[j // page], j % page] = c["vs"][b]
    o, lse = run(p4q, dev, c)
    reached = 0
    for b, n in enumerate(lens):
        if n <= 0:
            assert bool((o[b] == 0).all())
            continue
        k, v = (x[b].double().repeat_interleave(H // Hkv, 1) for x in (c["ks"], c["vs"]))  # [n, H, dh]
        s = torch.einsum("hd,lhd->lh", c["q"][b].double().view(H, dh), k) * dh ** -0.5
        weighs = (torch.exp(s - s.amax(0)) > 2.0 ** -100)[:, :, None]
        inf = v.abs() == math.inf
        want = torch.where(((v == math.inf) & weighs).any(0), math.inf, 0.0) + \
            torch.where(((v == -math.inf) & weighs).any(0), -math.inf, 0.0) + torch.where(torch.isnan(v).any(0), math.nan, 0.0)
        got = o[b].view(H, dh).double()
        special, left_out = ~torch.isfinite(want), (inf & ~weighs).any(0)
        same = (got == want) | (torch.isnan(got) & torch.isnan(want))
        wrong = special & ~left_out & ~same
        assert not bool(wrong.any()), f"sequence {b}: {int(wrong.sum())} of {int(special.sum())}, {got[wrong][:4].tolist()}"
        reached += int(special.sum())
        finite = torch.where(torch.isfinite(c["vs"][b]), c["vs"][b], torch.zeros((), dtype=c["vs"][b].dtype, device=dev))
        exact = torch.einsum("lh,lhd->hd", torch.softmax(s, 0), finite.double().repeat_interleave(H // Hkv, 1))
        row = torch.where(special | left_out, exact, got).to(o.dtype).view(1, H * dh)
        check({**c, "ks": [c["ks"][b]], "vs": [finite], "q": c["q"][b:b + 1]}, row, lse[b:b + 1])
    assert reached > 0


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("H,Hkv,dh,page", [(4, 4, 128, 16), (8, 2, 128, 4), (8, 1, 64, 16), (3, 1, 64, 2), (12, 1, 64, 16)])
def test_infinite_values_at_every_position(p4q, dev, dt, H, Hkv, dh, page):
    """One infinite value of each sign per sequence and head, at each position in turn; one NaN."""
    def put(b, v, g):
        n = v.shape[0]
        v[b % n, :, 5] = math.inf
        v[7 * b % n, :, 9] = -math.inf
        v[(b + 3) % n, 0, 11] = math.nan
        v[b % n, :, 20], v[(b + 1) % n, :, 20] = math.inf, -math.inf

    _non_finite(p4q, dev, [40] * 80, H, Hkv, dh, page, dt, put, seed=H)


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("dh", [64, 128])
def test_infinite_values_of_one_position(p4q, dev, dt, dh):
    """A weight of exactly 1."""
    def put(b, v, g):
        v[:, :, b::7] = math.inf
        v[:, :, b + 1::7] = -math.inf

    _non_finite(p4q, dev, [1, 1, 0, 1], 8, 2, dh, 16, dt, put)


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("lens,H,Hkv,qscale", [([9000], 32, 8, 1.0), ([700], 8, 8, 1.0), ([3000, 40, 2500], 16, 1, 1.0),
                                               ([300] * 9, 8, 2, 8.0), ([2100], 4, 1, 8.0), ([150] * 400, 4, 2, 3.0)])
def test_infinite_values_in_every_split(p4q, dev, dt, lens, H, Hkv, qscale):
    """Values anywhere in long and short sequences, of weights down to 2^-100 of the largest."""
    def put(b, v, g):
        n, heads, dh = v.shape
        at = torch.randint(0, n, (heads, dh), generator=g, device=v.device)
        sign = torch.randint(0, 3, (heads, dh), generator=g, device=v.device)
        what = torch.tensor([math.inf, -math.inf, 1.0], device=v.device)[sign].to(v.dtype)
        v.scatter_(0, at[None], what[None])

    _non_finite(p4q, dev, lens, H, Hkv, 128, 16, dt, put, qscale=qscale, seed=len(lens))


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("n", [1, 17, 300, 9000])
def test_a_row_of_scores_of_minus_infinity_is_empty(p4q, dev, dt, n):
    """No position has a weight: o = 0, also where values are infinite."""
    c = make(dev, [n, 5], 4, 2, 128, 16, dt, seed=n)
    c["q"][:] = 0
    c["q"][:, ::128] = 1.0
    for b in range(2):
        c["ks"][b][:, :, 0] = -math.inf
        c["vs"][b][:, :, 3] = math.inf
        j = torch.arange(c["ks"][b].shape[0], device=dev)
        at = c["table"][b].long()[j // 16], j % 16
        c["k"][at], c["v"][at] = c["ks"][b], c["vs"][b]
    o, lse = run(p4q, dev, c)
    assert bool((o == 0).all()) and bool((lse == -math.inf).all())
