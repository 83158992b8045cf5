"""Attention of one token for groups of sequences behind shared prefixes, against a
64-bit evaluation of the formula on the gathered positions.

Bound: that of the attention over a paged cache of 16 bits (vmax the largest |v| of the head's
positions): u |o| + 2 (d + a + 2^-19) vmax + 2^-25, d = 2^-23 (dh A + 2 S + 8) from a score
(A the largest sum |q_d k_d| scale, S the largest |score|), a = 2^-24 (64 + n / 16) from
adding n weights in parts; the logarithm of the sum d + a + 2^-22 |lse|."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DT = {"fp16": (torch.float16, 2.0 ** -11), "bf16": (torch.bfloat16, 2.0 ** -8)}
NAN = float("nan")


def make(dev, groups, H, Hkv, dh, page, dt, seed, order="slots", qscale=1.0, before=(), behind=(), vfill=None, cols=None):
    """groups: (prefix, [positions of each sequence behind it (negative: it ends before the prefix does)]);
    before, behind: lengths of sequences in no group. Slots that nothing should read hold NaN, and the columns
    before a prefix's end pages outside the cache, but for the group's first sequence."""
    g = torch.Generator(device=dev).manual_seed(seed)
    dtype = DT[dt][0]
    plan = [(n, 0, None) for n in before]  # (length, prefix, first of the group)
    starts = [len(plan)]
    for prefix, own in groups:
        first = len(plan)
        plan += [(prefix + x, prefix, first) for x in own]
        starts.append(len(plan))
    plan += [(n, 0, None) for n in behind]
    n = len(plan)
    longest = max(max(length, prefix) for length, prefix, _ in plan)
    cols = max(1, (longest + page - 1) // page) if cols is None else cols
    table = np.full((n, cols), 2 ** 30, np.int32)
    total = sum((max(0, x[0]) + x[1] + 2 * page) // page for x in plan) + 3
    free = list(torch.randperm(total, generator=g, device=dev).cpu().numpy())
    for b, (length, prefix, first) in enumerate(plan):
        lo = 0 if first in (None, b) else prefix // page
        hi = (max(length, prefix if first == b else 0) + page - 1) // page
        for col in range(lo, hi):
            table[b, col] = free.pop()
    shape = (total, page, Hkv, dh) if order != "heads" else (total, Hkv, page, dh)
    k, v = (torch.full(shape, NAN, dtype=dtype, device=dev) for _ in range(2))
    if order == "heads":
        k, v = k.transpose(1, 2), v.transpose(1, 2)

    def fill(row, lo, hi):
        j = torch.arange(lo, hi, device=dev)
        pg = torch.from_numpy(table[row]).to(dev).long()[j // page]
        kk, vv = (torch.randn((hi - lo, Hkv, dh), generator=g, device=dev).to(dtype) for _ in range(2))
        if vfill is not None:
            vv.fill_(vfill)
        k[pg, j % page], v[pg, j % page] = kk, vv
        return kk, vv

    ks, vs, shared = [], [], {}
    for b, (length, prefix, first) in enumerate(plan):
        length = max(0, length)
        if first is None:
            kk, vv = fill(b, 0, length)
        else:
            if first == b:
                shared[b] = fill(b, 0, prefix)
            kk, vv = (x[:length] for x in shared[first])
            if length > prefix:
                more = fill(b, prefix, length)
                kk, vv = torch.cat((kk, more[0])), torch.cat((vv, more[1]))
        ks.append(kk)
        vs.append(vv)
    q = (torch.randn((n, (H + 2 * Hkv) * dh), generator=g, device=dev) * qscale).to(dtype)[:, :H * dh]
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)  # noqa: E731
    return {"q": q, "k": k, "v": v, "table": torch.from_numpy(table).to(dev), "ks": ks, "vs": vs,
            "lens": i32([x[0] for x in plan]), "start": i32(starts), "prefix": i32([p for p, _ in groups]), "H": H,
            "Hkv": Hkv, "dh": dh, "dt": dt}


def workspace(p4q, dev, c):
    return p4q.prefix_attention_workspace(c["q"].shape[0], c["prefix"].shape[0], c["H"], c["dh"], dev)


def run(p4q, dev, c, ws=None, scale=None, pitch=8, status=0):
    n, cols = c["q"].shape
    if ws is None:
        ws = workspace(p4q, dev, c)
    o = torch.full((n, cols + pitch), 7.0, dtype=c["q"].dtype, device=dev)
    lse = torch.full((n, c["H"]), 7.0, device=dev)
    p4q.p4q_prefix_attention(c["q"], c["k"], c["v"], c["table"], c["lens"], c["start"], c["prefix"], o[:, :cols], ws,
                             scale=scale, lse=lse)
    torch.cuda.synchronize()
    assert p4q.p4q_device_status() == status
    assert bool((o[:, cols:] == 7.0).all()), "columns past the heads were written"
    return o[:, :cols], lse


def check(c, o, lse, scale=None, rows=None):
    H, Hkv, dh = c["H"], c["Hkv"], c["dh"]
    scale = dh ** -0.5 if scale is None else scale
    u = DT[c["dt"]][1]
    for b in range(len(c["ks"])) if rows is None else rows:
        k, v = c["ks"][b].double(), c["vs"][b].double()
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
        d = 2.0 ** -23 * (dh * A + 2 * S + 8)
        a = 2.0 ** -24 * (64 + k.shape[0] / 16)
        bound = u * want.abs() + 2 * (d + a + 2.0 ** -19)[:, None] * vmax[:, None] + 2.0 ** -25
        err = (got - want).abs()
        assert bool((err <= bound).all()), f"sequence {b}: {int((err > bound).sum())} off, {float((err / bound).max()):.3g} of the bound"
        lerr = (glse - wlse).abs()
        assert bool((lerr <= d + a + 2.0 ** -22 * wlse.abs()).all()), f"sequence {b}: lse off by {float(lerr.max()):.3g}"


HEADS = [(8, 8), (8, 2), (28, 4), (24, 2), (16, 1), (40, 1), (3, 3), (40, 8)]


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("dh", [128, 64])
@pytest.mark.parametrize("page", [16, 1, 8, 64, 256])
def test_prefixes_and_pages(p4q, dev, dt, dh, page):
    for i, groups in enumerate(([(1, [0])], [(127, [1, 0, 5]), (128, [2, 0]), (129, [300, 1, 1])], [(661, [5, 90, 17, 64, 1])],
                                [(256, [16] * 9), (16, [1]), (0, [30, 0, 2]), (1000, [1, 2, 200])])):
        H, Hkv = HEADS[(i + page + dh // 64) % len(HEADS)]
        c = make(dev, groups, H, Hkv, dh, page, dt, seed=i, order=("slots", "heads")[i % 2])
        check(c, *run(p4q, dev, c))


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("H,Hkv", HEADS)
def test_heads(p4q, dev, dt, H, Hkv):
    c = make(dev, [(333, [1, 50, 0, 200]), (40, [3] * 33)], H, Hkv, 128, 16, dt, seed=H)
    check(c, *run(p4q, dev, c))


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("groups,H,Hkv,dh,page,cols", [
    ([(20000, [100] * 3)], 8, 1, 128, 64, None), ([(30000, [1])], 1, 1, 64, 16, None),
    ([(3000, list(range(0, 600, 5)))], 24, 2, 64, 32, None), ([(500, [3] * 150)], 40, 2, 128, 16, None),
    ([(100 + 37 * i, [i % 3] * (1 + i % 4)) for i in range(70)], 8, 2, 128, 8, None), ([(700, [20] * 16)], 8, 8, 128, 16, 3000),
    ([(50, [4000, 1, 0, 3000])], 32, 8, 128, 16, None)])
def test_long_prefixes_and_many_sequences(p4q, dev, dt, groups, H, Hkv, dh, page, cols):
    c = make(dev, groups, H, Hkv, dh, page, dt, seed=3, cols=cols)
    o, lse = run(p4q, dev, c)
    check(c, o, lse)
    o2, lse2 = run(p4q, dev, c)
    assert torch.equal(o, o2) and torch.equal(lse, lse2), "two calls differ"


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
def test_short_sequences_and_ones_in_no_group(p4q, dev, dt):
    """Sequences that end before their group's prefix does, empty ones, the group's first among them."""
    c = make(dev, [(300, [-10, 5, -300, -299, 0, -301, 40]), (64, [-64, 3]), (20, [-5])], 8, 2, 128, 16, dt, seed=1,
             before=[70, 0], behind=[1, 333])
    check(c, *run(p4q, dev, c))


def test_a_prefix_of_nothing_is_paged_attention(p4q, dev):
    c = make(dev, [(0, [700, 30, 1])], 8, 2, 128, 16, "fp16", seed=2)
    o, lse = run(p4q, dev, c)
    check(c, o, lse)
    c["prefix"].fill_(-5)
    assert torch.equal(run(p4q, dev, c)[0], o)
    assert torch.equal(p4q.paged_attention(c["q"], c["k"], c["v"], c["table"], c["lens"]), o)


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
def test_sharp_scores_and_scales(p4q, dev, dt):
    for qscale, scale in ((30.0, None), (1.0, 3.0), (1.0, -0.1), (1.0, 0.0)):
        c = make(dev, [(1500, [300, 1, 20, 0]), (129, [2])], 8, 2, 128, 16, dt, seed=7, qscale=qscale)
        check(c, *run(p4q, dev, c, scale=scale), scale=scale)


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
def test_values_that_are_not_finite(p4q, dev, dt):
    c = make(dev, [(300, [20, 5, -150, 0])], 4, 2, 64, 16, dt, seed=4)
    table = c["table"]
    page = lambda b, j: (int(table[b, j // 16]), j % 16)  # noqa: E731
    c["v"][(*page(0, 200), 0, 7)] = float("inf")  # of the prefix, past the third's end
    c["vs"] = [x.clone() for x in c["vs"]]
    o, lse = run(p4q, dev, c)
    o = o.view(4, 4, 64)
    for b in (0, 1, 3):
        assert bool((o[b, :2, 7] == float("inf")).all())
        assert int(o[b].isfinite().sum()) == 4 * 64 - 2
    check(c, o.reshape(4, -1), lse, rows=[2])
    c["k"][(*page(0, 10), 1, 0)] = NAN
    c["q"] = c["q"].clone()
    c["q"][1, 0] = float("nan")
    o, lse = run(p4q, dev, c)
    o = o.view(4, 4, 64)
    assert bool(o[:, 2:].isnan().all()) and bool(lse[:, 2:].isnan().all())
    assert bool(o[1, 0].isnan().all()) and bool(lse[1, 0].isnan()) and bool(lse[0, :2].isfinite().all())


def test_scores_of_minus_infinity_have_no_weight(p4q, dev):
    c = make(dev, [(200, [10, 0, 3])], 4, 2, 64, 16, "bf16", seed=4)
    c["q"] = c["q"].clone().abs()
    c["k"].masked_fill_(c["k"].isfinite(), 0).nan_to_num_(nan=0.0)
    table = c["table"]
    c["ks"] = [torch.zeros_like(k) for k in c["ks"]]
    for j in range(150):  # of the prefix's positions only the last have a weight
        c["k"][int(table[0, j // 16]), j % 16, :, 0] = -float("inf")
    o, lse = run(p4q, dev, c)
    c["ks"], c["vs"] = [k[150:] for k in c["ks"]], [v[150:] for v in c["vs"]]
    check(c, o, lse)


def test_pages_groups_and_lengths_outside_their_ranges(p4q, dev):
    c = make(dev, [(200, [10, 30])], 4, 2, 64, 16, "fp16", seed=4)
    c["table"][0, 3] = 10 ** 6
    keep = [torch.arange(n, device=dev) for n in (210, 230)]
    keep = [x[(x < 48) | (x >= 64)] for x in keep]
    c["ks"], c["vs"] = ([x[i] for x, i in zip(y, keep)] for y in (c["ks"], c["vs"]))
    check(c, *run(p4q, dev, c, status=8))
    c["lens"][1] = 2 ** 31 - 1  # cut to the table's columns
    c["lens"].clamp_(max=2 ** 31 - 1)
    run(p4q, dev, c, status=8)
    for starts, prefix in (([0, 5], [200]), ([-1, 2], [200]), ([1, 0], [200]), ([0, 2], [10 ** 9]), ([2 ** 31 - 1, -2 ** 31], [7])):
        d = make(dev, [(200, [10, 30])], 4, 2, 64, 16, "fp16", seed=4)
        d["table"].clamp_(max=d["k"].shape[0] - 1)
        d["start"], d["prefix"] = (torch.tensor(x, dtype=torch.int32, device=dev) for x in (starts, prefix))
        run(p4q, dev, d, status=8)
    d = make(dev, [(64, [1, 2]), (32, [3, 4])], 4, 2, 64, 16, "fp16", seed=4)  # overlapping groups
    d["table"].clamp_(max=d["k"].shape[0] - 1)
    d["start"] = torch.tensor([2, 0, 4], dtype=torch.int32, device=dev)
    run(p4q, dev, d, status=8)


@pytest.mark.parametrize("page", [16, 8])
def test_offsets_past_32_bits(p4q, dev, page):
    dh, Hkv = 64, 2
    c = make(dev, [(70, [20, 5, -30]), (16, [9])], 8, Hkv, dh, page, "fp16", seed=12)
    pages = c["k"].shape[0]
    stride = (5 << 30) // (pages - 1) // 8 * 8  # elements: pages 5 G of them apart in all
    for name in ("k", "v"):
        room = torch.empty((stride * pages + page * Hkv * dh,), dtype=torch.float16, device=dev)
        far = room.as_strided((pages, page, Hkv, dh), (stride, Hkv * dh, dh, 1))
        far.copy_(c[name])
        c[name] = far
    check(c, *run(p4q, dev, c))


def test_graphs_and_streams(p4q, dev):
    """A captured call replayed on other lengths and prefixes, and two streams with a workspace each."""
    a = make(dev, [(700, [90, 3, 40])], 8, 2, 128, 16, "fp16", seed=1)
    b = make(dev, [(1300, [20] * 5), (40, [7])], 8, 2, 128, 16, "fp16", seed=2)
    want = [run(p4q, dev, c, pitch=0)[0].clone() for c in (a, b)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    ws = [workspace(p4q, dev, c) for c in (a, b)]
    outs = [torch.empty_like(c["q"]) for c in (a, b)]
    torch.cuda.synchronize()
    for _ in range(20):
        for c, s, w, o in zip((a, b), streams, ws, outs):
            p4q.p4q_prefix_attention(c["q"], c["k"], c["v"], c["table"], c["lens"], c["start"], c["prefix"], o, w, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1])
    o = torch.empty_like(a["q"])
    lens, prefix = a["lens"].clone(), a["prefix"].clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        p4q.p4q_prefix_attention(a["q"], a["k"], a["v"], a["table"], lens, a["start"], prefix, o, ws[0])
    g.replay()
    assert torch.equal(o, want[0])
    lens.copy_(torch.tensor([690, 703, 31], dtype=torch.int32))
    prefix.fill_(650)
    a["table"][1:, 650 // 16:700 // 16 + 1] = a["table"][0, 650 // 16:700 // 16 + 1]
    g.replay()
    other = run(p4q, dev, dict(a, lens=lens, prefix=prefix), pitch=0)[0]
    assert torch.equal(o, other) and not torch.equal(o, want[0])
    args = (b["q"], b["k"], b["v"], b["table"], b["lens"], b["start"], b["prefix"])
    assert torch.equal(p4q.prefix_attention(*args), want[1])
    s = torch.cuda.Stream()
    got = p4q.prefix_attention(*args, stream=s)
    s.synchronize()
    assert torch.equal(got, want[1])


def test_steps_back_to_back_on_one_workspace(p4q, dev):
    """Calls of different batches one after the other, nothing waited for in between."""
    cs = [make(dev, [(100 + 400 * i, [i, 50, 3]), (64, [9] * (i + 1))], 8, 2, 64, 16, "bf16", seed=i) for i in range(4)]
    want = [run(p4q, dev, c, pitch=0)[0].clone() for c in cs]
    ws = max((workspace(p4q, dev, c) for c in cs), key=lambda w: w.numel())
    outs = [torch.empty_like(c["q"]) for c in cs]
    for _ in range(10):
        for c, o in zip(cs, outs):
            p4q.p4q_prefix_attention(c["q"], c["k"], c["v"], c["table"], c["lens"], c["start"], c["prefix"], o, ws)
    torch.cuda.synchronize()
    for o, w in zip(outs, want):
        assert torch.equal(o, w)


def test_more_groups_than_a_warp_has_lanes(p4q, dev):
    c = make(dev, [(30 + 3 * i, [i % 4, 9][:1 + i % 2]) for i in range(100)], 8, 2, 64, 8, "bf16", seed=5, before=[20], behind=[5])
    check(c, *run(p4q, dev, c))
    c = make(dev, [(17, [2])] * 33 + [(900, [1, 30])], 4, 4, 128, 16, "fp16", seed=6)
    check(c, *run(p4q, dev, c))


@pytest.mark.parametrize("graph", [False, True])
def test_what_is_appended_just_before_is_seen(p4q, dev, graph):
    """Append and attention back to back, nothing in between: each step's rows lie in slots that the
    attention before has read as masked ones, on the same SMs perhaps."""
    steps, H, Hkv, dh, page = 24, 8, 4, 128, 32
    c = make(dev, [(200, [3, 40, 7, 0, 12])] * 3, H, Hkv, dh, page, "fp16", seed=8, cols=9)
    n = c["lens"].shape[0]
    free = torch.arange(c["k"].shape[0], c["k"].shape[0] + 2 * n, device=dev, dtype=torch.int32)
    k, v = (torch.cat((x, torch.zeros((2 * n, *x.shape[1:]), dtype=x.dtype, device=dev))).nan_to_num_(nan=3.0) for x in (c["k"], c["v"]))
    table = c["table"].clone()
    at = 0
    for b in range(n):  # pages for the steps to come
        for col in range(table.shape[1]):
            if (b % 5 == 0 or col >= 200 // page) and int(table[b, col]) >= k.shape[0] and at < free.numel() and col * page < int(c["lens"][b]) + steps:
                table[b, col] = free[at]
                at += 1
    g = torch.Generator(device=dev).manual_seed(1)
    rows = torch.randn((steps, n, (H + 2 * Hkv) * dh), generator=g, device=dev).half()
    one, zero = torch.ones((400, dh // 2), device=dev), torch.zeros((400, dh // 2), device=dev)
    lens = [c["lens"] + i + 1 for i in range(steps)]
    pos = [x - 1 for x in lens]
    outs = [torch.empty((n, H * dh), dtype=torch.float16, device=dev) for _ in range(steps)]
    ws = workspace(p4q, dev, c)

    def step(i, o):
        y = rows[i]
        q = y[:, :H * dh]
        p4q.p4q_rope_append(q, y[:, H * dh:(H + Hkv) * dh], y[:, (H + Hkv) * dh:], one, zero, pos[i], k, v, table, q)
        p4q.p4q_prefix_attention(q, k, v, table, lens[i], c["start"], c["prefix"], o, ws)

    def all_steps():
        for i in range(steps):
            step(i, outs[i])

    k0, v0 = k.clone(), v.clone()
    torch.cuda.synchronize()
    if graph:
        cg = torch.cuda.CUDAGraph()
        with torch.cuda.graph(cg):
            all_steps()
        cg.replay()
    else:
        all_steps()
    torch.cuda.synchronize()
    assert p4q.p4q_device_status() == 0
    k.copy_(k0)
    v.copy_(v0)
    for i in range(steps):  # the same, each step waited for
        want = torch.empty_like(outs[i])
        step(i, want)
        torch.cuda.synchronize()
        assert torch.equal(outs[i], want), f"step {i}"
