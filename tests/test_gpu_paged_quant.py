"""Attention of one token over a paged cache of codes, against a 64-bit evaluation of
the formula on the gathered positions' values code * scale.

Bound of an output element, vmax the largest |v| of the head's positions (full scale:
largest scale times 127 or 7):
  u |o| + 2 (d + a + 2^-19) vmax + 2^-25
with u the output type's unit roundoff (2^-11 fp16, 2^-8 bf16; 2^-25 for an fp16 output
below its normal range); d = 2^-23 (dh A + 4 S + 8) the relative error of a softmax
weight from its score (A the largest sum |q_d k_d| scale over the positions: dh additions
of fp32, each off by one place of a partial sum at most; S the largest |score|: three
factors, the exponent's difference; the exponential's own 2 places); a = 2^-24 (64 + n / 16)
from adding n weights in parts; and 2^-19 for weights times scales held in two fp16 values
(2^-21 of each, and 2^-35 of the largest one for each of up to 2^15 positions). The logarithm
of the sum: d + a + 2^-22 |lse|."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DT = {"fp16": (torch.float16, 2.0 ** -11), "bf16": (torch.bfloat16, 2.0 ** -8)}
NAN = float("nan")


def pack(c):
    return ((c[..., 0::2] & 15) | (c[..., 1::2] << 4)).view(torch.uint8)


def make(dev, lens, H, Hkv, dh, page, bits, dt, seed, order="slots", qscale=1.0, spread=0.5, cols=None):
    """Caches whose slots past the lengths (and pages of nobody) hold codes of every kind with scales NaN."""
    g = torch.Generator(device=dev).manual_seed(seed)
    dtype = DT[dt][0]
    n = len(lens)
    need = [(max(0, x) + page - 1) // page for x in lens]
    cols = max(1, max(need)) if cols is None else cols
    pages = sum(need) + 3
    perm = torch.randperm(pages, generator=g, device=dev).cpu().numpy()
    table = np.full((n, cols), 2 ** 30, np.int32)  # (past a sequence's pages: not to be read)
    at = 0
    for b in range(n):
        table[b, :need[b]] = perm[at:at + need[b]]
        at += need[b]
    most = 127 if bits == 8 else 7
    width, ct = (dh, torch.int8) if bits == 8 else (dh // 2, torch.uint8)
    if order == "heads":
        codes = [torch.full((pages, Hkv, page, width), 119, dtype=ct, device=dev).transpose(1, 2) for _ in range(2)]
        scales = [torch.full((pages, page, Hkv), NAN, device=dev) for _ in range(2)]
    else:
        pad = 16 if order == "padded" else 0
        codes = [torch.full((pages, page, Hkv, width + pad), 119, dtype=ct, device=dev)[..., :width] for _ in range(2)]
        scales = [torch.full((pages, Hkv, page + pad), NAN, device=dev)[..., :page].transpose(1, 2) for _ in range(2)]
    q = (torch.randn((n, (H + 2 * Hkv) * dh), generator=g, device=dev) * qscale).to(dtype)[:, :H * dh]  # rows with a pitch
    ks, vs = [], []
    for b, length in enumerate(lens):
        length = max(0, length)
        j = torch.arange(length, device=dev)
        pg = torch.from_numpy(table[b]).to(dev).long()[j // page]
        for c, sc, keep in zip(codes, scales, (ks, vs)):
            code = torch.randint(-most, most + 1, (length, Hkv, dh), generator=g, device=dev, dtype=torch.int8)
            s = 2.0 ** ((2 * torch.rand((length, Hkv), generator=g, device=dev) - 1) * spread) * 2.0 / most
            c[pg, j % page] = code if bits == 8 else pack(code)
            sc[pg, j % page] = s
            keep.append(code.double() * s.double()[..., None])
    return {"q": q, "cache": (*codes, *scales), "table": torch.from_numpy(table).to(dev), "ks": ks, "vs": vs,
            "lens": torch.tensor(lens, dtype=torch.int32, device=dev), "H": H, "Hkv": Hkv, "dh": dh, "dt": dt}


def run(p4q, dev, c, ws=None, scale=None, pitch=8, status=0):
    n, cols = c["q"].shape
    if ws is None:
        ws = p4q.paged_attention_workspace(dev)
    o = torch.full((n, cols + pitch), 7.0, dtype=c["q"].dtype, device=dev)
    lse = torch.full((n, c["H"]), 7.0, device=dev)
    p4q.p4q_paged_attention_quant(c["q"], *c["cache"], c["table"], c["lens"], o[:, :cols], ws, scale=scale, lse=lse)
    torch.cuda.synchronize()
    assert p4q.p4q_device_status() == status
    assert bool((o[:, cols:] == 7.0).all()), "columns past the heads were written"
    return o[:, :cols], lse


def check(c, o, lse, scale=None):
    H, Hkv, dh = c["H"], c["Hkv"], c["dh"]
    scale = dh ** -0.5 if scale is None else scale
    u = DT[c["dt"]][1]
    for b in range(len(c["ks"])):
        k, v = c["ks"][b], c["vs"][b]
        got, glse = o[b].double().view(H, dh), lse[b].double()
        if k.shape[0] == 0:
            assert bool((got == 0).all()) and bool((glse == -float("inf")).all())
            continue
        q = c["q"][b].double().view(Hkv, H // Hkv, dh)
        s = torch.einsum("hgd,lhd->hgl", q, k) * scale
        A = (torch.einsum("hgd,lhd->hgl", q.abs(), k.abs()) * abs(scale)).amax(-1).reshape(H)
        S = s.abs().amax(-1).reshape(H)
        want = torch.einsum("hgl,lhd->hgd", torch.softmax(s, -1), v).reshape(H, dh)
        wlse = torch.logsumexp(s, -1).reshape(H)
        vmax = v.abs().amax((0, 2)).repeat_interleave(H // Hkv)
        d = 2.0 ** -23 * (dh * A + 4 * S + 8)
        a = 2.0 ** -24 * (64 + k.shape[0] / 16)
        bound = u * want.abs() + 2 * (d + a + 2.0 ** -19)[:, None] * vmax[:, None] + 2.0 ** -25
        err = (got - want).abs()
        assert bool((err <= bound).all()), f"sequence {b}: {int((err > bound).sum())} off, {float((err / bound).max()):.3g} of the bound"
        lerr = (glse - wlse).abs()
        assert bool((lerr <= d + a + 2.0 ** -22 * wlse.abs()).all()), f"sequence {b}: lse off by {float(lerr.max()):.3g}"


HEADS = [(8, 8), (8, 2), (28, 4), (24, 2), (16, 1), (20, 1), (3, 3), (40, 8)]


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("page", [1, 2, 8, 16, 64, 256])
def test_lengths_and_pages(p4q, dev, bits, dt, dh, page):
    for i, lens in enumerate(([1], [0, 1, 2, 15, 16, 17], [63, 64, 65, 127, 128, 129, 255, 256, 257], [704, -3, 300])):
        H, Hkv = HEADS[(i + page + dh // 64 + bits) % len(HEADS)]
        c = make(dev, lens, H, Hkv, dh, page, bits, dt, seed=i, order=("slots", "heads", "padded")[i % 3])
        check(c, *run(p4q, dev, c))


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("H,Hkv", HEADS)
def test_heads(p4q, dev, bits, dt, H, Hkv):
    c = make(dev, [333, 17, 0, 1025], H, Hkv, 128, 16, bits, dt, seed=H)
    check(c, *run(p4q, dev, c))


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("lens,H,Hkv,dh,page,cols", [
    ([40000], 8, 1, 128, 64, None), ([9000, 1, 0, 20000, 512], 8, 2, 64, 16, None), ([5000] * 12, 32, 8, 128, 16, None),
    (list(range(1, 700, 5)), 8, 8, 64, 8, None), ([200] * 100, 8, 2, 128, 32, None), ([9, 700], 8, 2, 128, 16, 3000)])
def test_long_and_many_sequences(p4q, dev, bits, lens, H, Hkv, dh, page, cols):
    c = make(dev, lens, H, Hkv, dh, page, bits, "fp16" if bits == 8 else "bf16", seed=3, cols=cols)
    o, lse = run(p4q, dev, c)
    check(c, o, lse)
    o2, lse2 = run(p4q, dev, c)
    assert torch.equal(o, o2) and torch.equal(lse, lse2), "two calls differ"


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dt", ["fp16", "bf16"])
def test_sharp_scores_and_scales_of_many_sizes(p4q, dev, bits, dt):
    for qscale, spread, scale in ((30.0, 0.5, None), (1.0, 8.0, None), (0.01, 10.0, 3.0), (1.0, 0.5, -0.1), (1.0, 0.5, 0.0)):
        c = make(dev, [900, 70, 1], 8, 2, 128, 16, bits, dt, seed=7, qscale=qscale, spread=spread)
        check(c, *run(p4q, dev, c, scale=scale), scale=scale)


def test_scales_of_any_size_and_sign_of_bf16(p4q, dev):
    """Rows of tiny, huge and negative scales: outputs within a few roundings of their own size."""
    for size in (2.0 ** -100, 2.0 ** 60, -1.0):
        c = make(dev, [300, 5], 4, 2, 64, 16, 8, "bf16", seed=1)
        vs = c["cache"][3]
        vs.copy_(vs * size)
        c["vs"] = [v * size for v in c["vs"]]
        o, _ = run(p4q, dev, c)
        want = [torch.einsum("hgl,lhd->hgd", torch.softmax(torch.einsum("hgd,lhd->hgl", c["q"][b].double().view(2, 2, 64), k) / 8, -1),
                             v).reshape(-1) for b, (k, v) in enumerate(zip(c["ks"], c["vs"]))]
        for b in range(2):
            vmax = c["vs"][b].abs().max()
            assert bool(((o[b].double() - want[b]).abs() <= 2.0 ** -8 * want[b].abs() + 2.0 ** -17 * vmax).all())


def test_queries_of_any_size_of_bf16(p4q, dev):
    """q far outside fp16's range with keys as far on the other side: the scores are ordinary."""
    for size in (2.0 ** 70, 2.0 ** -70):
        c = make(dev, [300, 64], 4, 4, 128, 16, 4, "bf16", seed=2)
        c["q"] = (c["q"].float() * size).to(torch.bfloat16)
        c["cache"][2].copy_(c["cache"][2] / size)
        c["ks"] = [k / size for k in c["ks"]]
        check(c, *run(p4q, dev, c))


def test_values_that_are_not_finite(p4q, dev):
    c = make(dev, [100, 100, 100], 4, 2, 64, 16, 8, "fp16", seed=4)
    table, ks, vs = c["table"], c["cache"][2], c["cache"][3]
    page = lambda b, j: (int(table[b, j // 16]), j % 16)  # noqa: E731
    ks[(*page(0, 40), 0)] = NAN    # a key: all of its head
    vs[(*page(1, 40), 1)] = NAN    # a value
    vs[(*page(2, 99), 0)] = float("inf")
    o, lse = run(p4q, dev, c)
    o = o.view(3, 4, 64)
    assert bool(o[0, :2].isnan().all()) and bool(lse[0, :2].isnan().all())
    assert bool(o[1, 2:].isnan().all()) and bool(o[2, :2].isnan().all())
    assert bool(o[0, 2:].isfinite().all()) and bool(o[1, :2].isfinite().all()) and bool(o[2, 2:].isfinite().all())
    assert bool(lse[1:].isfinite().all())
    c["q"] = c["q"].clone()
    c["q"][0, 3] = NAN
    o, lse = run(p4q, dev, c)
    assert bool(o[0, :64].isnan().all()) and bool(lse[0, 0].isnan())


def test_pages_and_lengths_outside_the_cache(p4q, dev):
    c = make(dev, [100, 64, 40], 4, 2, 64, 16, 8, "fp16", seed=4)
    bad = c["table"].clone()
    bad[0, 2], bad[1, 0], bad[1, 3] = 10 ** 6, -1, 2 ** 31 - 1
    c["table"] = bad
    keep = [torch.arange(n, device=dev) for n in (100, 64, 40)]
    keep[0] = keep[0][(keep[0] < 32) | (keep[0] >= 48)]
    keep[1] = keep[1][(keep[1] >= 16) & (keep[1] < 48)]
    c["ks"] = [k[i] for k, i in zip(c["ks"], keep)]
    c["vs"] = [v[i] for v, i in zip(c["vs"], keep)]
    check(c, *run(p4q, dev, c, status=8))
    c = make(dev, [112, 64], 4, 2, 64, 16, 4, "fp16", seed=4)
    c["lens"][0] = 2 ** 31 - 1  # cut to the table
    check(c, *run(p4q, dev, c, status=8))


@pytest.mark.parametrize("bits", [4, 8])
def test_offsets_past_32_bits(p4q, dev, bits):
    lens, page, Hkv, dh = [90, 33], 16, 2, 128
    c = make(dev, lens, 8, Hkv, dh, page, bits, "fp16", seed=9)
    pages = c["cache"][0].shape[0]
    stride = (5 << 30) // (pages - 1) // 16 * 16  # pages 5 GB apart in all
    width = c["cache"][0].shape[-1]
    far = []
    for x in c["cache"][:2]:
        room = torch.empty((stride * pages + page * Hkv * width,), dtype=torch.uint8, device=dev).view(x.dtype)
        y = room.as_strided((pages, page, Hkv, width), (stride, Hkv * width, width, 1))
        y.copy_(x)
        far.append(y)
    sstride = (5 << 28) // (pages - 1)  # of elements: the scales' bytes pass 2^32 as well
    for x in c["cache"][2:]:
        room = torch.empty((sstride * pages + page * Hkv,), device=dev)
        y = room.as_strided((pages, page, Hkv), (sstride, 1, page))
        y.copy_(x)
        far.append(y)
    c["cache"] = tuple(far)
    check(c, *run(p4q, dev, c))


def test_graphs_and_streams(p4q, dev):
    """A captured step replayed on changed inputs, and two streams with a workspace each."""
    a = make(dev, [700, 90], 8, 2, 128, 16, 4, "fp16", seed=1)
    b = make(dev, [1300, 20], 8, 2, 128, 16, 4, "fp16", seed=2)
    want = [run(p4q, dev, c, pitch=0)[0].clone() for c in (a, b)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    ws = [p4q.paged_attention_workspace(dev) for _ in range(2)]
    outs = [torch.empty_like(a["q"]) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for c, s, w, o in zip((a, b), streams, ws, outs):
            p4q.p4q_paged_attention_quant(c["q"], *c["cache"], c["table"], c["lens"], o, w, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1])
    q, o = a["q"].clone(), torch.empty_like(a["q"])
    lens = a["lens"].clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        p4q.p4q_paged_attention_quant(q, *a["cache"], a["table"], lens, o, ws[0])
    g.replay()
    assert torch.equal(o, want[0])
    lens.copy_(torch.tensor([31, 90], dtype=torch.int32))
    g.replay()
    short = dict(a, lens=lens)
    assert torch.equal(o, run(p4q, dev, short, pitch=0)[0])
    assert torch.equal(p4q.paged_attention_quant(q, *a["cache"], a["table"], a["lens"]), want[0])


def test_a_cache_as_it_is_written(p4q, dev):
    """Append, then attend: against attention over the rows that the codes stand for, in a 16-bit cache's place."""
    g = torch.Generator(device=dev).manual_seed(8)
    n, H, Hkv, dh, page, S = 3, 8, 4, 128, 16, 200
    for bits in (4, 8):
        width, ct = (dh, torch.int8) if bits == 8 else (dh // 2, torch.uint8)
        cols = (S + page) // page
        cache = [torch.zeros((n * cols, page, Hkv, width), dtype=ct, device=dev) for _ in range(2)]
        cache += [torch.zeros((n * cols, page, Hkv), device=dev) for _ in range(2)]
        table = torch.randperm(n * cols, generator=g, device=dev).to(torch.int32).view(n, cols)
        y = torch.randn((n * S, (H + 2 * Hkv) * dh), generator=g, device=dev).half()
        q, k, v = y[:, :H * dh], y[:, H * dh:(H + Hkv) * dh], y[:, (H + Hkv) * dh:]
        ang = torch.rand((S, dh // 2), generator=g, device=dev) * 6
        pos = torch.arange(S, dtype=torch.int32, device=dev).repeat(n)
        seq = torch.arange(n, dtype=torch.int32, device=dev).repeat_interleave(S)
        k_out, v_out, q_out = (torch.empty((n * S, w), dtype=torch.float16, device=dev) for w in (Hkv * dh, Hkv * dh, H * dh))
        p4q.p4q_rope_append_quant(q, k, v, ang.cos(), ang.sin(), pos, *cache, table, q_out, k_out=k_out, v_out=v_out, seq=seq)
        last = q_out.view(n, S, H * dh)[:, -1].contiguous()
        lens = torch.full((n,), S, dtype=torch.int32, device=dev)
        o = p4q.paged_attention_quant(last, *cache, table, lens).double().view(n, H, dh)
        kk, vv = (x.double().view(n, S, Hkv, dh).repeat_interleave(H // Hkv, 2) for x in (k_out, v_out))
        s = torch.einsum("nhd,nlhd->nhl", last.double().view(n, H, dh), kk) / dh ** 0.5
        want = torch.einsum("nhl,nlhd->nhd", torch.softmax(s, -1), vv)
        # the rows are the codes' values rounded to fp16: 2^-11 of each k (its score's error e with weights off
        # by 2 e at most) and of each v
        e = 2.0 ** -11 * (torch.einsum("nhd,nlhd->nhl", last.double().view(n, H, dh).abs(), kk.abs()) / dh ** 0.5).amax(-1, keepdim=True)
        vmax = vv.abs().amax((1, 3))[..., None]
        assert bool(((o - want).abs() <= 2.0 ** -11 * want.abs() + (2.2 * e + 2.0 ** -11 + 2.0 ** -16) * vmax).all())
