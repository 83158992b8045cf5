"""The position rotation and the append to a paged cache, against a 64-bit
evaluation of the same formula.

Bound: c, s are given; two products and a sum in fp32 have an error of at most
4 * 2^-24 (|x_a| + |x_b|), the rounding to the output type at most u |y| (u = 2^-11
for fp16, 2^-8 for bf16) or, for an fp16 value below its normal range, 2^-25. What is
copied has to be equal, and slots that no token names stay as they were."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DT = {"fp16": (torch.float16, 2.0 ** -11), "bf16": (torch.bfloat16, 2.0 ** -8)}
FILL = 7.0


def make_cache(dev, pages, page, Hkv, dh, dtype, order="slots"):
    if order == "slots":  # [pages, slots, heads, dh]
        c = [torch.full((pages, page, Hkv, dh), FILL, dtype=dtype, device=dev) for _ in range(2)]
    elif order == "heads":  # heads before slots in memory
        c = [torch.full((pages, Hkv, page, dh), FILL, dtype=dtype, device=dev).transpose(1, 2) for _ in range(2)]
    else:  # keys and values of a slot side by side, rows padded
        both = torch.full((pages, page, Hkv, 2, dh + 8), FILL, dtype=dtype, device=dev)
        c = [both[..., 0, :dh], both[..., 1, :dh]]
    return c


def rotate(x, cos, sin, rot, inter):
    """x [T, heads, dh] float64; cos, sin [T, rot/2]."""
    y = x.copy()
    i = np.arange(rot // 2)
    a, b = (2 * i, 2 * i + 1) if inter else (i, i + rot // 2)
    c, s = cos[:, None, :], sin[:, None, :]
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    size = np.abs(x)
    both = np.zeros_like(x)
    both[..., a] = both[..., b] = size[..., a] + size[..., b]
    return y, both


def close(got, want, both, dt):
    u = DT[dt][1]
    bound = u * np.abs(want) + 4 * 2.0 ** -24 * both + (2.0 ** -25 if dt == "fp16" else 0.0)
    err = np.abs(got.astype(np.float64) - want)
    assert np.all(err <= bound), f"{np.sum(err > bound)} off, largest error {err.max():.3g}"


def run_case(p4q, dev, T, seqs, H, Hkv, dh, rot, inter, dt, page, order="slots", k_rows=True, in_place=False, seed=0,
             use_seq=True, use_rot_pos=True):
    rng = np.random.default_rng(seed)
    dtype = DT[dt][0]
    cols = 6
    table = rng.permutation(seqs * cols + 5)[:seqs * cols].astype(np.int32).reshape(seqs, cols)
    room = cols * page
    # distinct (sequence, position) pairs, positions across the whole table
    if use_seq:
        pick = rng.choice(seqs * room, size=T, replace=False)
        seq, pos = (pick // room).astype(np.int32), (pick % room).astype(np.int32)
    else:
        seq, pos = np.arange(T, dtype=np.int32), rng.integers(0, room, T).astype(np.int32)
    max_pos = 3 * room + 1
    rp = rng.integers(0, max_pos, T).astype(np.int32) if use_rot_pos else pos
    ang = rng.uniform(-np.pi, np.pi, (max_pos, rot // 2))
    cos, sin = np.cos(ang).astype(np.float32), np.sin(ang).astype(np.float32)
    pad = 8
    fused = torch.from_numpy(rng.standard_normal((T, (H + 2 * Hkv) * dh + pad)).astype(np.float32)).to(dev).to(dtype)
    q, k, v = fused[:, :H * dh], fused[:, H * dh:(H + Hkv) * dh], fused[:, (H + Hkv) * dh:(H + 2 * Hkv) * dh]
    q0, k0, v0 = (x.double().cpu().numpy().reshape(T, -1, dh) for x in (q, k, v))
    kc, vc = make_cache(dev, seqs * cols + 5, page, Hkv, dh, dtype, order)
    if in_place:
        q_out, k_out = q, k if k_rows else None
    else:
        q_out = torch.full((T, H * dh + pad), FILL, dtype=dtype, device=dev)[:, :H * dh]
        k_out = torch.full((T, Hkv * dh + pad), FILL, dtype=dtype, device=dev)[:, :Hkv * dh] if k_rows else None
    up = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(dev)  # noqa: E731
    p4q.p4q_rope_append(q, k, v, up(cos), up(sin), up(pos), kc, vc, up(table), q_out, k_out=k_out,
                        seq=up(seq) if use_seq else None, rot_pos=up(rp) if use_rot_pos else None, interleaved=inter)
    torch.cuda.synchronize()
    assert p4q.p4q_device_status() == 0
    c64, s64 = cos.astype(np.float64)[rp], sin.astype(np.float64)[rp]
    wq, bq = rotate(q0, c64, s64, rot, inter)
    wk, bk = rotate(k0, c64, s64, rot, inter)
    got_q = q_out.double().cpu().numpy().reshape(T, H, dh)
    close(got_q, wq, bq, dt)
    assert np.array_equal(got_q[..., rot:], q0[..., rot:])
    page_of, slot = table[seq, pos // page], pos % page
    gk, gv = kc.double().cpu().numpy(), vc.double().cpu().numpy()
    close(gk[page_of, slot], wk, bk, dt)
    assert np.array_equal(gk[page_of, slot][..., rot:], k0[..., rot:])
    assert np.array_equal(gv[page_of, slot], v0)
    for g in (gk, gv):
        left = np.ones(g.shape[:2], bool)
        left[page_of, slot] = False
        assert np.all(g[left] == FILL), "a slot of no token was written"
    if k_rows:
        gko = k_out.double().cpu().numpy().reshape(T, Hkv, dh)
        assert np.array_equal(gko, gk[page_of, slot])
    if order == "beside":
        base = kc._base if kc._base is not None else kc
        assert bool((base[..., dh:] == FILL).all()), "padding beside the rows was written"
    if not in_place:
        assert bool((fused[:, -pad:] == fused[:, -pad:]).all())
        assert np.array_equal(v.double().cpu().numpy().reshape(T, Hkv, dh), v0)


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("T,seqs,H,Hkv,dh,rot,inter,page", [
    (1, 1, 1, 1, 128, 128, False, 16), (1, 1, 32, 32, 128, 128, False, 16), (3, 2, 5, 1, 64, 64, True, 1),
    (33, 4, 8, 2, 128, 64, False, 8), (130, 7, 28, 4, 128, 128, True, 64), (257, 3, 40, 40, 128, 128, False, 32),
    (64, 2, 7, 7, 64, 16, False, 128), (19, 1, 12, 3, 64, 32, True, 4), (700, 5, 40, 8, 128, 112, False, 256),
    (2500, 6, 3, 1, 64, 64, False, 128),
])
def test_rotation_and_append(p4q, dev, dt, T, seqs, H, Hkv, dh, rot, inter, page):
    run_case(p4q, dev, T, seqs, H, Hkv, dh, rot, inter, dt, page, seed=T + H)


@pytest.mark.parametrize("order", ["slots", "heads", "beside"])
@pytest.mark.parametrize("k_rows,in_place,use_seq,use_rot_pos", [(True, True, True, True), (False, False, False, True),
                                                                 (True, False, False, False), (False, True, True, False)])
def test_layouts_and_options(p4q, dev, order, k_rows, in_place, use_seq, use_rot_pos):
    run_case(p4q, dev, 24, 24, 8, 4, 128, 128, False, "fp16", 16, order, k_rows, in_place, 5, use_seq, use_rot_pos)
    run_case(p4q, dev, 24, 24, 8, 4, 64, 32, True, "bf16", 8, order, k_rows, in_place, 6, use_seq, use_rot_pos)


def _small(dev, T=4, seqs=4, cols=2, page=16, pages=8):
    g = torch.Generator(device=dev).manual_seed(1)
    r = lambda c: torch.randn((T, c * 128), generator=g, device=dev).half()  # noqa: E731
    kc, vc = make_cache(dev, pages, page, 2, 128, torch.float16)
    return {"q": r(4), "k": r(2), "v": r(2), "cos": torch.ones((64, 64), device=dev), "sin": torch.zeros((64, 64), device=dev),
            "pos": torch.arange(T, dtype=torch.int32, device=dev) * 5, "k_cache": kc, "v_cache": vc,
            "table": torch.arange(seqs * cols, dtype=torch.int32, device=dev).view(seqs, cols),
            "q_out": torch.full((T, 512), FILL, dtype=torch.float16, device=dev)}


def test_padding_tokens_write_nothing(p4q, dev):
    a = _small(dev)
    a["pos"][2] = -1
    p4q.p4q_rope_append(**a)
    torch.cuda.synchronize()
    assert p4q.p4q_device_status() == 0
    assert bool((a["q_out"][2] == FILL).all())
    assert bool((a["k_cache"][4:6] == FILL).all()) and bool((a["v_cache"][4:6] == FILL).all())
    for t in (0, 1, 3):
        assert bool((a["q_out"][t] == a["q"][t]).all())
        assert bool((a["v_cache"][2 * t, 5 * t] == a["v"][t].view(2, 128)).all())


@pytest.mark.parametrize("what,value", [("pos", 32), ("pos", 2 ** 31 - 1), ("rot_pos", 64), ("rot_pos", -1), ("seq", 4),
                                        ("seq", -1), ("table", 8), ("table", -1), ("table", 2 ** 31 - 1)])
def test_an_index_outside_its_table_is_reported(p4q, dev, what, value):
    """Token 1 has it: nothing of that token is written, the others are done."""
    a = _small(dev)
    a["rot_pos"] = torch.zeros(4, dtype=torch.int32, device=dev)
    a["seq"] = torch.arange(4, dtype=torch.int32, device=dev)
    if what == "table":
        a["table"][1, 0] = value
    else:
        a[what][1] = value
    p4q.p4q_rope_append(**a)
    assert p4q.p4q_device_status() == 8
    assert p4q.p4q_device_status() == 0
    assert bool((a["q_out"][1] == FILL).all())
    assert bool((a["k_cache"][2:4] == FILL).all()) and bool((a["v_cache"][2:4] == FILL).all())
    for t in (0, 2, 3):
        assert bool((a["q_out"][t] == a["q"][t]).all())
        assert bool((a["k_cache"][2 * t, 5 * t] == a["k"][t].view(2, 128)).all())


def test_a_cache_past_32_bit_offsets(p4q, dev):
    a = _small(dev)
    stride = 1 << 28  # elements between pages: the last page starts past 2^32 bytes and 2^31 elements
    big = [torch.empty((9 * stride + (1 << 14),), dtype=torch.float16, device=dev) for _ in range(2)]
    kc, vc = (b.as_strided((10, 16, 2, 128), (stride, 256, 128, 1)) for b in big)
    kc[9].fill_(FILL)
    vc[9].fill_(FILL)
    a["table"].fill_(9)
    a["k_cache"], a["v_cache"] = kc, vc
    p4q.p4q_rope_append(**a)
    torch.cuda.synchronize()
    assert p4q.p4q_device_status() == 0
    for t in range(4):
        assert bool((kc[9, 5 * t] == a["k"][t].view(2, 128)).all())
        assert bool((vc[9, 5 * t] == a["v"][t].view(2, 128)).all())
    assert bool((kc[9, 1:5] == FILL).all())


def test_non_finite_rows_stay_their_own(p4q, dev):
    """An infinite or NaN value of one pair reaches that pair only (and v as it is)."""
    a = _small(dev)
    clean = _small(dev)
    a["q"][0, 3] = float("nan")
    a["k"][1, 130] = float("inf")
    a["v"][2, 7] = float("nan")
    p4q.p4q_rope_append(**a)
    p4q.p4q_rope_append(**clean)
    torch.cuda.synchronize()
    q, w = a["q_out"], clean["q_out"]
    same = q == w
    assert bool((~same[0]).sum() <= 2) and not bool(same[0, 3]) and bool(same[1:].all())
    k, w = a["k_cache"], clean["k_cache"]
    assert int((k != w).sum()) <= 2 and bool(torch.isinf(k[2, 5, 1, 2]))
    v, w = a["v_cache"], clean["v_cache"]
    assert int((v != w).sum()) == 1 and bool(torch.isnan(v[4, 10, 0, 7]))


def test_another_stream_and_a_graph(p4q, dev):
    a, b = _small(dev), _small(dev)
    p4q.p4q_rope_append(**a)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        p4q.p4q_rope_append(**b)
    s.synchronize()
    assert bool((a["q_out"] == b["q_out"]).all()) and bool((a["k_cache"] == b["k_cache"]).all())
    c = _small(dev)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p4q.p4q_rope_append(**c)
    c["pos"].add_(1)  # read when the graph runs
    graph.replay()
    torch.cuda.synchronize()
    for t in range(4):
        at = 5 * t + 1
        assert bool((c["v_cache"][2 * t + at // 16, at % 16] == c["v"][t].view(2, 128)).all())


def test_the_binding_refuses(p4q, dev):
    a = _small(dev)
    bad = [("q", a["q"].bfloat16(), TypeError), ("q", a["q"].t(), TypeError), ("k", a["k"][:, :128], ValueError),
           ("v", a["v"][:2], ValueError), ("pos", a["pos"].long(), TypeError), ("pos", a["pos"][:2], ValueError),
           ("pos", None, TypeError), ("cos", a["cos"].half(), TypeError), ("cos", a["cos"][:32], ValueError),
           ("table", a["table"].long(), TypeError), ("v_cache", a["v_cache"].transpose(1, 2), TypeError),
           ("v_cache", a["v_cache"].bfloat16(), TypeError), ("k_cache", a["k_cache"].float(), TypeError),
           ("q_out", a["q_out"][:, :256], ValueError), ("q", a["q"][:, :500], ValueError)]
    for name, value, error in bad:
        with pytest.raises(error):
            p4q.p4q_rope_append(**{**a, name: value})
    with pytest.raises(p4q.P4QError):  # more tokens than sequences without seq
        p4q.p4q_rope_append(**{**a, "table": a["table"][:2]})
    torch.cuda.synchronize()
    assert bool((a["q_out"] == FILL).all()) and bool((a["k_cache"] == FILL).all())
