"""The rotation and the append to a cache of codes, against the definition in numpy:
rotation with each product and the sum rounded to fp32, then to the rows' type; per
token and head a = max |x|, s = fl32(a / m), codes round_half_even(fl32(x / s)). All
of it is defined bit for bit, so everything has to be equal; slots that no token
names stay as they were."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DT = {"fp16": torch.float16, "bf16": torch.bfloat16}
FILL, SFILL = 85, 7.0


def make_cache(dev, pages, page, Hkv, dh, bits, order="slots"):
    """Codes and scales of keys and values, filled."""
    width, dt = (dh, torch.int8) if bits == 8 else (dh // 2, torch.uint8)
    if order == "slots":
        c = [torch.full((pages, page, Hkv, width), FILL, dtype=dt, device=dev) for _ in range(2)]
        s = [torch.full((pages, Hkv, page), SFILL, device=dev).transpose(1, 2) for _ in range(2)]
    elif order == "heads":
        c = [torch.full((pages, Hkv, page, width), FILL, dtype=dt, device=dev).transpose(1, 2) for _ in range(2)]
        s = [torch.full((pages, page, Hkv), SFILL, device=dev) for _ in range(2)]
    else:  # keys and values of a slot side by side, rows padded; scales in one array
        both = torch.full((pages, page, Hkv, 2, width + 16), FILL, dtype=dt, device=dev)
        c = [both[..., 0, :width], both[..., 1, :width]]
        sc = torch.full((pages, 2, Hkv, page + 1), SFILL, device=dev)
        s = [sc[:, i, :, :page].transpose(1, 2) for i in range(2)]
    return (*c, *s)


def to_rows(x, dtype):
    return torch.from_numpy(np.ascontiguousarray(x)).to(dtype)


def rotate(x, cos, sin, rot, inter, dtype):
    """x [T, heads, dh] fp32 -> rows of dtype, as fp32; every operation rounded to fp32."""
    y = x.copy()
    i = np.arange(rot // 2)
    a, b = (2 * i, 2 * i + 1) if inter else (i, i + rot // 2)
    c, s = cos[:, None, :], sin[:, None, :]
    with np.errstate(invalid="ignore", over="ignore"):
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
    assert y.dtype == np.float32
    return to_rows(y, dtype).float().numpy()


def quantise(x, bits):
    """Rows x [T, heads, dh] fp32 -> codes int8, scales fp32."""
    m = np.float32(127 if bits == 8 else 7)
    a = np.abs(x).max(-1)
    bad = ~np.isfinite(x).all(-1)
    a = np.where(bad, np.float32(0), a).astype(np.float32)
    s = a / m
    x = np.where(bad[..., None], np.float32(0), x)
    code = np.rint(x / np.where(s > 0, s, np.float32(1))[..., None]).astype(np.float32)
    assert np.abs(code).max(initial=0) <= m
    return code.astype(np.int8), np.where(bad, np.float32(np.nan), s)


def unpack(c, bits):
    c = c.cpu().numpy()
    if bits == 8:
        return c
    w = np.stack((c & 15, c >> 4), -1).reshape(*c.shape[:-1], -1).astype(np.int16)
    return np.where(w > 7, w - 16, w).astype(np.int8)


def same(got, want):
    np.testing.assert_array_equal(np.asarray(got, np.float64), np.asarray(want, np.float64))


def run_case(p4q, dev, T, seqs, H, Hkv, dh, rot, inter, dt, bits, page, order="slots", rows=True, in_place=False, seed=0,
             use_seq=True, use_rot_pos=True, spread=0.0, special=False):
    rng = np.random.default_rng(seed)
    dtype = DT[dt]
    cols = 6
    table = rng.permutation(seqs * cols + 5)[:seqs * cols].astype(np.int32).reshape(seqs, cols)
    room = cols * page
    if use_seq:
        pick = rng.choice(seqs * room, size=T, replace=False)
        seq, pos = (pick // room).astype(np.int32), (pick % room).astype(np.int32)
    else:
        seq, pos = np.arange(T, dtype=np.int32), rng.integers(0, room, T).astype(np.int32)
    if special and T > 2:
        pos[1] = -1  # padding
    max_pos = 3 * room + 1
    rp = rng.integers(0, max_pos, T).astype(np.int32) if use_rot_pos else pos
    ang = rng.uniform(-np.pi, np.pi, (max_pos, rot // 2))
    cos, sin = np.cos(ang).astype(np.float32), np.sin(ang).astype(np.float32)
    x = rng.standard_normal((T, H + 2 * Hkv, dh)) * 2.0 ** rng.uniform(-spread, spread, (T, H + 2 * Hkv, 1))
    if special:  # rows of zeros, ties, one value, values that are not finite, the least ones
        for i in range(T):
            r = x[i, H + i % (2 * Hkv)]
            kind = i % 7
            if kind == 0:
                r[:] = 0
            elif kind == 1:  # quotients at halves: a = 127 or 7 units
                r[:] = rng.integers(-14, 15, dh) / 2
                r[0] = 127 if bits == 8 else 7
            elif kind == 2:
                r[dh // 2] = np.inf
            elif kind == 3:
                r[-1] = np.nan
            elif kind == 4:
                r[:] = 0
                r[3] = -1.5
            elif kind == 5:
                r[:] = np.round(r * 2) * (2.0 ** -24 if dt == "fp16" else 2.0 ** -133)
            else:
                r[::2] = r.max() / 2
    fused = to_rows(np.pad(x.reshape(T, -1), ((0, 0), (0, 8))), dtype).to(dev)
    q, k, v = fused[:, :H * dh], fused[:, H * dh:(H + Hkv) * dh], fused[:, (H + Hkv) * dh:(H + 2 * Hkv) * dh]
    q0, k0, v0 = (y.float().cpu().numpy().reshape(T, -1, dh) for y in (q, k, v))
    cache = make_cache(dev, seqs * cols + 5, page, Hkv, dh, bits, order)
    new = lambda n: torch.full((T, n + 8), SFILL, dtype=dtype, device=dev)[:, :n]  # noqa: E731
    q_out, k_out, v_out = (q, k, v) if in_place else (new(H * dh), new(Hkv * dh), new(Hkv * dh))
    if rows in (False, "v"):
        k_out = None
    if rows in (False, "k"):
        v_out = None
    up = lambda y: torch.from_numpy(np.ascontiguousarray(y)).to(dev)  # noqa: E731
    p4q.p4q_rope_append_quant(q, k, v, up(cos), up(sin), up(pos), *cache, up(table), q_out, k_out=k_out, v_out=v_out,
                              seq=up(seq) if use_seq else None, rot_pos=up(rp) if use_rot_pos else None, interleaved=inter)
    torch.cuda.synchronize()
    assert p4q.p4q_device_status() == 0
    done = pos >= 0
    at = np.where(done, rp, 0)
    kept = lambda want, old: np.where(done[:, None, None], want, old)  # noqa: E731
    old = (q0, k0, v0) if in_place else [np.full_like(y, SFILL) for y in (q0, k0, v0)]
    same(q_out.float().cpu().reshape(T, H, dh), kept(rotate(q0, cos[at], sin[at], rot, inter, dtype), old[0]))
    page_of, slot = table[np.where(done, seq, 0), np.where(done, pos, 0) // page], pos % page
    for name, r, codes, scales, out, before in (
            ("k", rotate(k0, cos[at], sin[at], rot, inter, dtype), cache[0], cache[2], k_out, old[1]),
            ("v", v0, cache[1], cache[3], v_out, old[2])):
        code, scale = quantise(r, bits)
        want = np.full((*codes.shape[:3], dh), 0, np.int8)
        got = unpack(codes, bits)
        touched = np.zeros(codes.shape[:2], bool)
        touched[page_of[done], slot[done]] = True
        want[page_of[done], slot[done]] = code[done]
        same(got[touched], want[touched])
        assert bool((codes.cpu().numpy()[~touched] == FILL).all()), "slots of no token were written"
        ws = np.full(scales.shape, SFILL, np.float32)
        ws[page_of[done], slot[done]] = scale[done]
        same(scales.cpu(), ws)
        if out is not None:
            value = to_rows(code.astype(np.float32) * scale[..., None], dtype).float().numpy()
            same(out.float().cpu().reshape(T, Hkv, dh), kept(value, before))


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("H,Hkv,dh,rot,inter", [(8, 8, 128, 128, False), (8, 2, 64, 64, True), (28, 4, 128, 64, False),
                                                (5, 5, 64, 32, False), (24, 2, 64, 16, True), (40, 40, 128, 128, True)])
def test_codes_are_equal(p4q, dev, bits, dt, H, Hkv, dh, rot, inter):
    for T, page, order in ((1, 16, "slots"), (3, 8, "heads"), (97, 1, "padded"), (700, 64, "slots")):
        run_case(p4q, dev, T, max(1, T // 3 + (page == 1) * T), H, Hkv, dh, rot, inter, dt, bits, page, order, seed=T,
                 spread=6.0 if dt == "fp16" else 60.0)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dt", ["fp16", "bf16"])
def test_ties_zeros_and_values_that_are_not_finite(p4q, dev, bits, dt):
    run_case(p4q, dev, 300, 60, 8, 4, 128, 128, False, dt, bits, 16, special=True, seed=5)
    run_case(p4q, dev, 300, 60, 4, 4, 64, 64, True, dt, bits, 16, special=True, seed=6)


@pytest.mark.parametrize("bits", [4, 8])
def test_in_place_without_rows_and_defaults(p4q, dev, bits):
    run_case(p4q, dev, 77, 20, 8, 4, 128, 128, False, "fp16", bits, 16, in_place=True)
    run_case(p4q, dev, 77, 20, 8, 4, 64, 64, False, "bf16", bits, 16, in_place=True, rows=False, special=True)
    run_case(p4q, dev, 33, 33, 8, 4, 128, 64, True, "bf16", bits, 32, rows=False, use_seq=False, use_rot_pos=False)
    run_case(p4q, dev, 33, 40, 1, 1, 128, 128, False, "fp16", bits, 32, use_seq=False)


@pytest.mark.parametrize("H,Hkv", [(40, 40), (1, 1), (33, 11), (3, 1), (128, 2)])
def test_rows_of_keys_or_values_alone(p4q, dev, H, Hkv):
    """Heads of q, k and v that a thread goes through one after the other, wherever its share begins."""
    for rows in ("k", "v"):
        run_case(p4q, dev, 70, 20, H, Hkv, 128, 128, False, "fp16", 4, 16, rows=rows)
        run_case(p4q, dev, 70, 20, H, Hkv, 64, 32, True, "bf16", 8, 8, rows=rows, in_place=True)


def test_every_pair_of_fp16_values_of_a_row(p4q, dev):
    """All quotients x / a of 2000 fp16 maxima a (those with ties among them) with 126 x each."""
    rng = np.random.default_rng(11)
    a = np.concatenate((np.arange(1, 1000), 2.0 ** rng.uniform(-14, 15, 1001))).astype(np.float16)
    k = a[:, None].astype(np.float64) * rng.uniform(-1, 1, (2000, 128))
    half = rng.integers(-127, 128, (2000, 128)) | 1
    k[:, ::3] = (a[:, None] * half / 254.0)[:, ::3]  # near and at codes + 1/2
    k[:, 1::3] = (a[:, None] * (half % 15 | 1) / 14.0)[:, 1::3]
    k = np.clip(k, -a[:, None].astype(np.float64), a[:, None])
    k[:, 0] = a
    rows = to_rows(k, torch.float16)
    dev_rows = rows.to(dev)
    T = 2000
    one, zero = torch.ones((T, 8), device=dev), torch.zeros((T, 8), device=dev)
    i32 = lambda n: torch.arange(n, dtype=torch.int32, device=dev)  # noqa: E731
    for bits in (4, 8):
        cache = make_cache(dev, T // 16, 16, 1, 128, bits)
        p4q.p4q_rope_append_quant(dev_rows, dev_rows, dev_rows, one, zero, i32(T), *cache, i32(T // 16).view(1, -1),
                                  torch.empty_like(dev_rows), seq=torch.zeros((T,), dtype=torch.int32, device=dev))
        code, scale = quantise(rows.float().numpy()[:, None], bits)
        for c, s in ((cache[0], cache[2]), (cache[1], cache[3])):
            same(unpack(c, bits).reshape(T, 1, 128), code)
            same(s.cpu().reshape(T, 1), scale)


def test_tokens_with_indices_outside_their_tables_are_not_written(p4q, dev):
    T, H, dh, page = 8, 2, 64, 16
    cache = make_cache(dev, 8, page, 2, dh, 8)
    before = [c.clone() for c in cache]
    table = torch.tensor([[0, 1], [2, 99], [-5, 3]], dtype=torch.int32, device=dev)
    q = torch.ones((T, H * dh), device=dev).half()
    q_out = torch.full_like(q, SFILL)
    cos = torch.ones((64, 32), device=dev)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=dev)  # noqa: E731
    #        padding, past the table, a page outside, a negative one, a sequence outside, rotation outside, good, good
    pos = i32(-1, 32, 16, 0, 3, 3, 5, 31)
    seq = i32(0, 0, 1, 2, 3, 0, 0, 0)
    rot = i32(0, 0, 0, 0, 0, 64, 63, 1)
    p4q.p4q_rope_append_quant(q, q, q, cos, cos, pos, *cache, table, q_out, seq=seq, rot_pos=rot)
    assert p4q.p4q_device_status() == 8  # P4Q_ERR_INDEX
    assert p4q.p4q_device_status() == 0
    assert bool((q_out[:6] == SFILL).all()) and bool((q_out[6:] != SFILL).all())
    for c, b in zip(cache, before):
        changed = (c != b).flatten(2).any(-1)
        want = torch.zeros_like(changed)
        want[0, 5] = want[1, 15] = True
        assert torch.equal(changed, want)


@pytest.mark.parametrize("bits", [4, 8])
def test_offsets_past_32_bits(p4q, dev, bits):
    """The codes of a cache whose pages lie 5 GB apart in all are those of a small one."""
    T, H, dh, page, pages = 90, 4, 128, 16, 9
    near = make_cache(dev, pages, page, H, dh, bits)
    width = near[0].shape[-1]
    stride, sstride = (5 << 30) // (pages - 1) // 16 * 16, (5 << 28) // (pages - 1)
    far = [torch.empty((stride * pages,), dtype=torch.uint8, device=dev).view(near[0].dtype).as_strided(
        (pages, page, H, width), (stride, H * width, width, 1)) for _ in range(2)]
    far += [torch.empty((sstride * pages,), device=dev).as_strided((pages, page, H), (sstride, 1, page)) for _ in range(2)]
    for x, y in zip(far, near):
        x.copy_(y)
    g = torch.Generator(device=dev).manual_seed(3)
    q = torch.randn((T, 3 * H * dh), generator=g, device=dev).half()
    ang = torch.rand((128, 64), generator=g, device=dev)
    pos = torch.arange(T, dtype=torch.int32, device=dev)
    table = torch.tensor([[8, 3, 7, 0, 5, 2]], dtype=torch.int32, device=dev)
    for cache in (near, far):
        p4q.p4q_rope_append_quant(*q.split(H * dh, 1), ang.cos(), ang.sin(), pos, *cache, table, torch.empty_like(q[:, :H * dh]),
                                  seq=torch.zeros_like(pos))
    assert p4q.p4q_device_status() == 0
    for x, y in zip(far, near):
        assert torch.equal(x, y)


def test_no_tokens_is_no_work(p4q, dev):
    cache = make_cache(dev, 2, 16, 2, 64, 4)
    q = torch.ones((0, 128), device=dev).half()
    cos = torch.ones((4, 32), device=dev)
    none = torch.zeros((0,), dtype=torch.int32, device=dev)
    before = p4q.p4q_launch_count()
    p4q.p4q_rope_append_quant(q, q, q, cos, cos, none, *cache, torch.zeros((1, 1), dtype=torch.int32, device=dev), q)
    assert p4q.p4q_launch_count() == before
