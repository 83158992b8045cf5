"""Attention of one token over a paged cache, against a 64-bit evaluation of the
formula on the gathered positions.

Bound of an output element, vmax the largest |v| of the head's positions:
  u |o| + 2 (d + a + 2^-19) vmax + 2^-25
with u the output type's unit roundoff (2^-11 fp16, 2^-8 bf16; 2^-25 for an fp16
output below its normal range); d = 2^-23 (dh A + 2 S + 8) the relative error of a
softmax weight from its score (A the largest sum |q_d k_d| scale over the positions:
dh additions of fp32, each off by one place of a partial sum at most; S the largest
|score|: the exponent's product and difference; the exponential's own 2 places);
a = 2^-24 (64 + n / 16) from adding n weights in parts; and 2^-19 for weights held
in two 16-bit values. The logarithm of the sum: d + a + 2^-22 |lse|."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DT = {"fp16": (torch.float16, 2.0 ** -11), "bf16": (torch.bfloat16, 2.0 ** -8)}


def make(dev, lens, H, Hkv, dh, page, dt, seed, order="slots", qscale=1.0, stale=float("nan"), cols=None):
    """Caches whose slots past the lengths (and pages of nobody) hold `stale`."""
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
    shape = (pages, page, Hkv, dh) if order != "heads" else (pages, Hkv, page, dh)
    k, v = (torch.full(shape, stale, dtype=dtype, device=dev) for _ in range(2))
    if order == "heads":
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    rows = torch.randn((n, (H + 2 * Hkv) * dh), generator=g, device=dev) * qscale
    q = rows.to(dtype)[:, :H * dh]  # rows with a pitch
    ks, vs = [], []
    for b, length in enumerate(lens):
        length = max(0, length)
        kk, vv = (torch.randn((length, Hkv, dh), generator=g, device=dev).to(dtype) for _ in range(2))
        j = torch.arange(length, device=dev)
        pg = torch.from_numpy(table[b]).to(dev).long()[j // page]
        k[pg, j % page], v[pg, j % page] = kk, vv
        ks.append(kk)
        vs.append(vv)
    return {"q": q, "k": k, "v": v, "table": torch.from_numpy(table).to(dev), "ks": ks, "vs": vs,
            "lens": torch.tensor(lens, dtype=torch.int32, device=dev), "H": H, "Hkv": Hkv, "dh": dh, "dt": dt}


def run(p4q, dev, c, ws=None, scale=None, pitch=8):
    n, cols = c["q"].shape
    if ws is None:
        ws = p4q.paged_attention_workspace(dev)
    o = torch.full((n, cols + pitch), 7.0, dtype=c["q"].dtype, device=dev)
    lse = torch.full((n, c["H"]), 7.0, device=dev)
    p4q.p4q_paged_attention(c["q"], c["k"], c["v"], c["table"], c["lens"], o[:, :cols], ws, scale=scale, lse=lse)
    torch.cuda.synchronize()
    assert p4q.p4q_device_status() == 0
    assert bool((o[:, cols:] == 7.0).all()), "columns past the heads were written"
    return o[:, :cols], lse


def check(c, o, lse, scale=None):
    H, Hkv, dh = c["H"], c["Hkv"], c["dh"]
    scale = dh ** -0.5 if scale is None else scale
    u = DT[c["dt"]][1]
    for b in range(len(c["ks"])):
        k, v = c["ks"][b].double(), c["vs"][b].double()
        got, glse = o[b].double().view(H, dh), lse[b].double()
        if k.shape[0] == 0:
            assert bool((got == 0).all()) and bool((glse == -float("inf")).all())
            continue
        q = c["q"][b].double().view(Hkv, H // Hkv, dh)
        s = torch.einsum("hgd,lhd->hgl", q, k) * scale
        A = (torch.einsum("hgd,lhd->hgl", q.abs(), k.abs()) * abs(scale)).amax(-1).reshape(H)
        want = torch.einsum("hgl,lhd->hgd", torch.softmax(s, -1), v).reshape(H, dh)
        wlse = torch.logsumexp(s, -1).reshape(H)
        n = k.shape[0]
        d = 2.0 ** -23 * (dh * A + 2 * s.abs().amax(-1).reshape(H) + 8)
        a = 2.0 ** -24 * (64 + n / 16)
        vmax = v.abs().amax((0, 2)).repeat_interleave(H // Hkv)
        bound = u * want.abs() + (2 * (d + a + 2.0 ** -19) * vmax + 2.0 ** -25)[:, None]
        err = (got - want).abs()
        assert bool((err <= bound).all()), f"sequence {b} ({n} positions): {int((err > bound).sum())} off, " \
                                           f"largest {float(err.max()):.3g}"
        lerr = (glse - wlse).abs()
        assert bool((lerr <= d + a + 2.0 ** -22 * wlse.abs()).all()), f"lse of {b}: {float(lerr.max()):.3g}"


EDGES = [0, 1, 2, 7, 8, 9, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 511, 513]


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("page", [1, 2, 8, 16, 64, 512])
@pytest.mark.parametrize("H,Hkv,dh", [(4, 4, 128), (8, 2, 64)])
def test_lengths_around_every_edge(p4q, dev, dt, page, H, Hkv, dh):
    c = make(dev, EDGES, H, Hkv, dh, page, dt, seed=page)
    check(c, *run(p4q, dev, c))


@pytest.mark.parametrize("H,Hkv", [(1, 1), (2, 1), (3, 1), (28, 4), (8, 1), (9, 1), (24, 2), (16, 1), (17, 1), (40, 1),
                                   (96, 2), (40, 40)])
@pytest.mark.parametrize("dh", [64, 128])
def test_head_groups(p4q, dev, H, Hkv, dh):
    for dt in ("fp16", "bf16"):
        c = make(dev, [700, 0, 33, 1500], H, Hkv, dh, 16, dt, seed=H)
        check(c, *run(p4q, dev, c))


@pytest.mark.parametrize("n,longest,H,Hkv,dh,page,dt", [
    (1, 20011, 32, 8, 128, 64, "bf16"), (1, 40000, 4, 1, 128, 16, "fp16"), (2, 33333, 8, 8, 64, 8, "fp16"),
    (160, 300, 8, 8, 128, 16, "fp16"), (700, 40, 16, 2, 64, 8, "bf16"), (33, 2500, 40, 8, 128, 32, "bf16"),
    (1, 1, 1, 1, 64, 1, "fp16"), (5000, 3, 2, 2, 128, 2, "fp16"),
])
def test_long_and_many(p4q, dev, n, longest, H, Hkv, dh, page, dt):
    rng = np.random.default_rng(n)
    lens = [longest] + [int(x) for x in (longest * rng.random(n - 1) ** 2)]
    c = make(dev, lens, H, Hkv, dh, page, dt, seed=longest)
    check(c, *run(p4q, dev, c))


@pytest.mark.parametrize("H,Hkv", [(40, 40), (32, 8), (24, 2), (8, 1)])
@pytest.mark.parametrize("longest", [1, 63, 65, 129, 250, 500, 704, 1100, 2300])
def test_few_sequences(p4q, dev, H, Hkv, longest):
    """One to a few sequences, as long as the table and much shorter, of each number of CTAs per key/value head."""
    for lens, dh, page, dt in (([longest], 128, 16, "fp16"), ([longest], 64, 8, "bf16"), ([longest, 0, 1], 128, 64, "bf16"),
                               ([longest, longest // 2, longest // 9, 66, 0], 64, 16, "fp16"),
                               ([longest // 3] * 9 + [longest], 128, 16, "fp16")):
        c = make(dev, [min(n, longest) for n in lens], H, Hkv, dh, page, dt, seed=longest)
        check(c, *run(p4q, dev, c))


@pytest.mark.parametrize("qscale,scale", [(30.0, None), (0.01, None), (1.0, 0.7), (1.0, -0.3), (1.0, 0.0)])
def test_peaked_flat_and_scaled(p4q, dev, qscale, scale):
    """One position dominates (its place varies), equal weights, other scales."""
    for dt in ("fp16", "bf16"):
        c = make(dev, [5, 130, 3000, 0, 777], 8, 2, 128, 16, dt, seed=3, qscale=qscale)
        check(c, *run(p4q, dev, c, scale=scale), scale=scale)


def test_rising_and_falling_scores(p4q, dev):
    """Scores that rise (or fall) along the cache by far more than an exponential's range."""
    for sign in (1.0, -1.0):
        c = make(dev, [2000], 4, 1, 128, 16, "bf16", seed=9)
        ramp = torch.linspace(-40, 40, 2000, device=dev)[:, None, None] * sign
        c["ks"][0][:] = (c["ks"][0].float() * 0.05 + ramp).bfloat16()
        j = torch.arange(2000, device=dev)
        pg = c["table"][0].long()[j // 16]
        c["k"][pg, j % 16] = c["ks"][0]
        c["q"][:] = (c["q"].float() * 0.01 + 0.4).bfloat16()
        check(c, *run(p4q, dev, c))


@pytest.mark.parametrize("order", ["slots", "heads"])
@pytest.mark.parametrize("page", [4, 16, 128])
def test_orders_of_slots_and_heads(p4q, dev, order, page):
    c = make(dev, [300, 17, 129], 12, 3, 128, page, "fp16", seed=2, order=order)
    check(c, *run(p4q, dev, c))


@pytest.mark.parametrize("stale", [float("nan"), float("inf"), -65504.0, 65504.0])
def test_what_lies_past_a_length_reaches_nothing(p4q, dev, stale):
    for dh in (64, 128):
        c = make(dev, [1, 5, 16, 100, 250, 0], 8, 2, dh, 32, "fp16", seed=4, stale=stale)
        check(c, *run(p4q, dev, c))


def test_negative_lengths_are_empty(p4q, dev):
    c = make(dev, [-3, 20, -2 ** 31], 8, 8, 128, 16, "fp16", seed=4)
    check(c, *run(p4q, dev, c))


def test_one_workspace_for_calls_of_any_sizes(p4q, dev):
    """The workspace is ready for the next call, whatever its sizes, without clearing."""
    ws = p4q.paged_attention_workspace(dev)
    cs = [make(dev, [9000], 32, 8, 128, 16, "bf16", 1), make(dev, [3] * 40, 8, 8, 64, 16, "fp16", 2),
          make(dev, [5000, 100, 7000], 16, 1, 128, 64, "fp16", 3), make(dev, [20000], 2, 2, 64, 8, "bf16", 4)]
    for i in (0, 1, 2, 3, 2, 1, 0, 3, 0, 2):
        check(cs[i], *run(p4q, dev, cs[i], ws))


def test_the_same_call_gives_the_same_bits(p4q, dev):
    ws = p4q.paged_attention_workspace(dev)
    c = make(dev, [9000, 40, 3000, 1], 32, 8, 128, 16, "bf16", 1)
    o, lse = run(p4q, dev, c, ws)
    for _ in range(20):
        o2, lse2 = run(p4q, dev, c, ws)
        assert torch.equal(o.view(torch.int16) if o.is_contiguous() else o.contiguous().view(torch.int16),
                           o2.contiguous().view(torch.int16))
        assert torch.equal(lse, lse2)


def test_pages_outside_the_cache_are_masked_and_reported(p4q, dev):
    for value in (-1, 2 ** 31 - 1, "pages"):
        c = make(dev, [200, 90], 8, 2, 128, 16, "fp16", seed=6)
        c["table"][0, 3] = c["k"].shape[0] if value == "pages" else value
        o = torch.empty_like(c["q"], memory_format=torch.contiguous_format)
        lse = torch.empty((2, 8), device=dev)
        p4q.p4q_paged_attention(c["q"], c["k"], c["v"], c["table"], c["lens"], o, p4q.paged_attention_workspace(dev), lse=lse)
        assert p4q.p4q_device_status() == 8
        assert p4q.p4q_device_status() == 0
        keep = torch.cat((torch.arange(0, 48), torch.arange(64, 200))).to(dev)
        c["ks"][0], c["vs"][0] = c["ks"][0][keep], c["vs"][0][keep]
        check(c, o, lse)


def test_a_length_past_the_table_is_cut_and_reported(p4q, dev):
    c = make(dev, [200, 90], 8, 2, 128, 16, "fp16", seed=6, cols=13)
    c["table"][1, :] = c["table"][0, :]
    c["lens"][0] = 2 ** 31 - 1
    o = torch.empty_like(c["q"], memory_format=torch.contiguous_format)
    lse = torch.empty((2, 8), device=dev)
    c["table"][0, 12] = c["table"][0, 0]  # columns 0 .. 12: 208 positions
    c["table"][1, :] = c["table"][0, :]
    p4q.p4q_paged_attention(c["q"], c["k"], c["v"], c["table"], c["lens"], o, p4q.paged_attention_workspace(dev), lse=lse)
    assert p4q.p4q_device_status() == 8
    kk, vv = c["ks"][0], c["vs"][0]
    c["ks"] = [torch.cat((kk[:192], kk[:16])), kk[:90]]
    c["vs"] = [torch.cat((vv[:192], vv[:16])), vv[:90]]
    check(c, o, lse)


def test_a_cache_past_32_bit_offsets(p4q, dev):
    c = make(dev, [70], 4, 2, 128, 16, "fp16", seed=8)
    stride = 1 << 28
    pages = c["k"].shape[0]
    big = [torch.empty((10 * stride + (1 << 14),), dtype=torch.float16, device=dev) for _ in range(2)]
    k, v = (b.as_strided((11, 16, 2, 128), (stride, 256, 128, 1)) for b in big)
    for i, p in enumerate(c["table"][0, :5].tolist()):
        k[10 - i].copy_(c["k"][p])
        v[10 - i].copy_(c["v"][p])
        c["table"][0, i] = 10 - i
    assert pages < 11
    c["k"], c["v"] = k, v
    check(c, *run(p4q, dev, c))


def test_infinite_keys_and_values_of_the_sequence(p4q, dev):
    """A score of -inf has no weight; one infinite value makes its column infinite, of its head only."""
    c = make(dev, [300, 300], 4, 4, 128, 16, "fp16", seed=12)
    ref, rlse = run(p4q, dev, c)
    q0 = c["q"][0, :128]
    d = int(q0.float().abs().argmax())
    bad = c["ks"][0].clone()
    bad[37, 0, d] = -float("inf") if float(q0[d]) > 0 else float("inf")
    c["k"][c["table"][0].long()[37 // 16], 37 % 16] = bad[37]
    big = c["vs"][1].clone()
    big[200, 3, 5] = float("inf")
    c["v"][c["table"][1].long()[200 // 16], 200 % 16] = big[200]
    o, lse = run(p4q, dev, c)
    keep = torch.cat((torch.arange(0, 37), torch.arange(38, 300))).to(dev)
    h0 = {**c, "H": 1, "Hkv": 1, "q": c["q"][:1, :128], "ks": [c["ks"][0][keep][:, :1]], "vs": [c["vs"][0][keep][:, :1]]}
    check(h0, o[:1, :128], lse[:1, :1])
    assert torch.equal(o[0, 128:], ref[0, 128:])
    same = o[1] == ref[1]
    assert bool(torch.isinf(o[1, 3 * 128 + 5])) and int((~same).sum()) == 1
    assert torch.equal(lse[1], rlse[1])


def test_another_stream_and_a_graph(p4q, dev):
    c = make(dev, [5000, 900], 32, 8, 128, 16, "bf16", 1)
    o, lse = run(p4q, dev, c)
    ws = p4q.paged_attention_workspace(dev)
    o2, lse2 = torch.empty_like(o), torch.empty_like(lse)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        for _ in range(3):
            p4q.p4q_paged_attention(c["q"], c["k"], c["v"], c["table"], c["lens"], o2, ws, lse=lse2)
    s.synchronize()
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p4q.p4q_paged_attention(c["q"], c["k"], c["v"], c["table"], c["lens"], o2, ws, lse=lse2)
    c["lens"][0] = 4321  # read when the graph runs
    c["lens"][1] = 0
    c["ks"], c["vs"] = [c["ks"][0][:4321], c["ks"][1][:0]], [c["vs"][0][:4321], c["vs"][1][:0]]
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    check(c, o2, lse2)


def test_the_binding_refuses(p4q, dev):
    c = make(dev, [20, 30], 8, 2, 128, 16, "fp16", 1)
    ws = p4q.paged_attention_workspace(dev)
    o = torch.full((2, 1024), 7.0, dtype=torch.float16, device=dev)
    a = dict(q=c["q"], k_cache=c["k"], v_cache=c["v"], table=c["table"], lens=c["lens"], o=o, ws=ws)
    for name, value, error in [("q", c["q"].float(), TypeError), ("q", c["q"][:1], ValueError),
                               ("q", c["q"][:, :1000], ValueError), ("o", o.bfloat16(), TypeError),
                               ("lens", c["lens"].long(), TypeError), ("lens", c["lens"][:1], ValueError),
                               ("lens", None, TypeError), ("ws", None, TypeError), ("ws", ws.cpu(), TypeError),
                               ("ws", ws[:-1], p4q.P4QError), ("lse", torch.empty((2, 4), device=dev), ValueError),
                               ("scale", float("nan"), p4q.P4QError), ("k_cache", c["k"][..., :96], TypeError)]:
        with pytest.raises(error):
            p4q.p4q_paged_attention(**{**a, name: value})
    c3 = make(dev, [20, 30], 6, 3, 128, 16, "fp16", 1)
    with pytest.raises(p4q.P4QError):  # 8 heads over 3
        p4q.p4q_paged_attention(**{**a, "k_cache": c3["k"], "v_cache": c3["v"]})
    torch.cuda.synchronize()
    assert bool((o == 7.0).all())
