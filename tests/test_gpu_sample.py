"""The draw of a token from logits, against the definition in 64 bits.

The kernel's weights come from fp32 exponentials. A weight w = 2^31 e, e = exp(-d),
differs from the 64-bit one by at most (3 d + 4) 2^-24 e 2^31 + 1 (d: a difference, the
reciprocal of T and a product, each rounded; e: two places; and the rounding to an
integer). So a sum of weights is off by at most the sum of these; the interval of the
drawn token, widened by that, has to hold u, and a token near a cut may be kept or
not where its sum or its exponential lies that near the cut. Where all weights are
exact (equal logits, or far apart ones) the token is one and the same."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def reference(x, T, top_k, top_p, min_p):
    """-> (order, kept bounds, e, d) of one row in 64 bits; x float64 without NaN, T > 0."""
    mx = x.max()
    with np.errstate(invalid="ignore"):
        d = np.where(x == mx, 0.0, (mx - x) / T)
    e = np.exp(-d)
    order = np.lexsort((np.arange(x.size), -x))
    return order, e, d


def slack(e, d):
    """Most that the kernel's weight may be off, in units of 1 = exp(0)."""
    fin = np.where(np.isfinite(d), d, 0.0)
    return (3 * fin + 4) * 2.0 ** -24 * e + 2.0 ** -31


def check_row(x, u, token, logprob, T=1.0, top_k=0, top_p=1.0, min_p=0.0):
    x = np.where(np.isnan(x), -np.inf, x.astype(np.float64))
    V = x.size
    if np.all(x == -np.inf):
        assert token == -1 and logprob == -np.inf
        return
    if not T > 0:
        assert token == int(np.argmax(x)) and logprob == 0.0
        return
    order, e, d = reference(x, T, top_k, top_p, min_p)
    es, sl = e[order], slack(e, d)[order]
    k = top_k if 0 < top_k < V else V
    es, sl, order = es[:k], sl[:k], order[:k]
    assert 0 <= token < V
    place = np.nonzero(order == token)[0]
    assert place.size == 1, f"token {token} is outside the first {k}"
    place = int(place[0])
    lo = hi = k  # the cut lies at some n with lo <= n <= hi
    if top_p < 1:
        need = max(top_p * es.sum(), 0.0)
        off = 2 * sl.sum() + 2.0 ** -30
        mass = np.cumsum(es)
        lo = int(np.searchsorted(mass, need - off)) + 1
        hi = min(k, int(np.searchsorted(mass, need + off)) + 1)
    if min_p > 0:
        mp = min(min_p, 1.0)
        lo = min(lo, int(np.sum(es - sl >= mp)) if mp < 1 else int(np.sum(es == 1.0)))
        hi = min(hi, int(np.sum(es + sl >= mp)))
    lo = max(1, min(lo, hi))
    assert place < hi, f"token {token} at place {place} is past the cut ({lo} .. {hi})"
    # its interval by index, for the shortest and the longest possible cut
    ok = False
    for n in {lo, hi} | set(range(lo, min(hi, lo + 64) + 1)):
        if place >= n:
            continue
        kept = np.sort(order[:n])
        w = e[kept]
        c = np.cumsum(w)
        at = int(np.searchsorted(kept, token))
        total, off = c[-1], slack(e, d)[kept].sum() * 2 + 2.0 ** -30
        a, b = (c[at] - w[at] - off) / total, (c[at] + off) / total
        if a <= min(max(u, 0.0), 1.0) <= b:
            ok = True
            want = -d[token] - math.log(total)
            bound = (3 * d[token] + 4) * 2.0 ** -24 + off / total + 2.0 ** -22 * (1 + abs(want))
            assert abs(logprob - want) <= bound or lo != hi, (logprob, want)
            break
    assert ok, f"u = {u} is not in the interval of token {token}"


def draw(p4q, dev, x, u, **params):
    """x [rows, V] torch on dev; u, params: numpy or None."""
    up = {k: None if v is None else torch.from_numpy(np.asarray(v)).to(dev) for k, v in params.items()}
    token, logprob = p4q.sample(x, torch.from_numpy(np.asarray(u, np.float32)).to(dev), **up)
    torch.cuda.synchronize()
    assert p4q.p4q_device_status() == 0
    return token.cpu().numpy(), logprob.cpu().numpy()


def logits(dev, rows, V, dt, seed, ld=None, spread=2.5):
    g = torch.Generator(device=dev).manual_seed(seed)
    x = torch.randn((rows, ld or V), generator=g, device=dev) * spread
    top = torch.randint(0, V, (rows, min(V, 20)), generator=g, device=dev)
    x.scatter_add_(1, top, torch.rand(top.shape, generator=g, device=dev) * 8)
    return x.to(dt)[:, :V]


TYPES = [torch.float16, torch.bfloat16, torch.float32]


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("V,ld", [(1, 1), (2, 2), (3, 5), (31, 31), (33, 40), (1000, 1001), (4096, 4096), (8191, 8193),
                                  (32000, 32000), (32003, 32064), (50001, 50001), (131071, 131076), (262144, 262144)])
def test_every_mode(p4q, dev, dt, V, ld):
    rows = 6
    x = logits(dev, rows, V, dt, seed=V, ld=ld)
    rng = np.random.default_rng(V)
    u = rng.random(rows).astype(np.float32)
    T = rng.uniform(0.3, 1.7, rows).astype(np.float32)
    k = rng.integers(1, max(2, min(V, 300)), rows).astype(np.int32)
    p = rng.uniform(0.3, 0.995, rows).astype(np.float32)
    m = rng.uniform(0.001, 0.3, rows).astype(np.float32)
    xs = x.float().cpu().numpy()
    for params in ({}, {"temperature": T}, {"top_k": k}, {"top_p": p}, {"min_p": m}, {"temperature": T, "top_k": k, "top_p": p},
                   {"temperature": T, "top_k": k, "top_p": p, "min_p": m}, {"top_p": p, "min_p": m}):
        token, lp = draw(p4q, dev, x, u, **params)
        for n in range(rows):
            one = {key: params[src][n] for key, src in (("T", "temperature"), ("top_k", "top_k"), ("top_p", "top_p"),
                                                        ("min_p", "min_p")) if src in params}
            check_row(xs[n], float(u[n]), int(token[n]), float(lp[n]), **one)


@pytest.mark.parametrize("spread", [0.3, 1.0, 6.0])
@pytest.mark.parametrize("V", [700, 20001, 131071, 262143])
def test_flat_and_peaked_rows(p4q, dev, V, spread):
    """Many tokens within reach of a cut, and few; top-k and the filters of each size."""
    rows = 12
    x = logits(dev, rows, V, torch.float32, seed=V + int(10 * spread), spread=spread)
    xs = x.cpu().numpy()
    rng = np.random.default_rng(V)
    u = rng.random(rows).astype(np.float32)
    k = np.array([1, 2, 30, 400, 511, 512, 513, 690, 5, 60, 700, 100], np.int32)
    p = np.array([0.05, 0.5, 0.9, 0.99, 0.999, 0.3, 0.8, 0.95, 0.7, 0.6, 0.9999, 0.2], np.float32)
    m = np.array([0.5, 0.1, 1e-3, 1e-5, 0.9, 0.01, 3e-4, 0.2, 0.05, 1e-4, 0.3, 2e-3], np.float32)
    for params in ({"top_k": k}, {"top_p": p}, {"min_p": m}, {"top_k": k, "top_p": p}, {"top_p": p, "min_p": m},
                   {"top_k": k, "min_p": m}, {"top_k": k, "top_p": p, "min_p": m}):
        token, lp = draw(p4q, dev, x, u, **params)
        for n in range(rows):
            check_row(xs[n], float(u[n]), int(token[n]), float(lp[n]), **{key: val[n] for key, val in params.items()})


def test_parameters_at_and_past_their_ends(p4q, dev):
    V = 3001
    nan, inf = float("nan"), float("inf")
    cases = [dict(T=0.0), dict(T=-1.0), dict(T=nan), dict(T=1e-30), dict(T=1e30), dict(T=inf), dict(top_k=0),
             dict(top_k=-5), dict(top_k=1), dict(top_k=V), dict(top_k=V + 1), dict(top_k=V - 1), dict(top_p=0.0),
             dict(top_p=-1.0), dict(top_p=1.0), dict(top_p=2.0), dict(top_p=nan), dict(top_p=1e-30), dict(min_p=0.0),
             dict(min_p=-1.0), dict(min_p=1.0), dict(min_p=3.0), dict(min_p=nan), dict(top_k=5, top_p=0.9999999)]
    x = logits(dev, len(cases), V, torch.float32, seed=3)
    xs = x.cpu().numpy()
    u = np.random.default_rng(0).random(len(cases)).astype(np.float32)
    get = lambda key, off, dt: np.array([c.get(key, off) for c in cases], dt)  # noqa: E731
    token, lp = draw(p4q, dev, x, u, temperature=get("T", 1.0, np.float32), top_k=get("top_k", 0, np.int32),
                     top_p=get("top_p", 1.0, np.float32), min_p=get("min_p", 0.0, np.float32))
    for n, c in enumerate(cases):
        c = {key: (v if v == v or key == "T" else {"top_p": 1.0, "min_p": 0.0}[key]) for key, v in c.items()}
        if c.get("T") == inf:
            c["T"] = 1e38
        check_row(xs[n], float(u[n]), int(token[n]), float(lp[n]), **c)


def test_uniform_numbers_at_and_past_their_ends(p4q, dev):
    V = 2000
    us = np.array([0.0, 1.0 - 2.0 ** -24, 1.0, 1.5, -0.5, float("nan"), 1e-40, 0.5], np.float32)
    x = torch.zeros((len(us), V), dtype=torch.float16, device=dev)  # equal weights: token floor(u V)
    token, lp = draw(p4q, dev, x, us)
    total = V * 2 ** 31
    want = [min(total - 1, max(0, math.floor(float(v) * total) if v == v else 0)) // 2 ** 31 for v in us]
    assert token.tolist() == want
    assert np.allclose(lp, -math.log(V), atol=1e-6)


@pytest.mark.parametrize("dt", TYPES)
def test_equal_logits_go_by_index(p4q, dev, dt):
    """All weights 2^31: cuts and draws are exact, ties to the lower index."""
    for V in (7, 1024, 5000, 70001):
        ks = [1, 2, 5, V // 2 + 1, V - 1, 0]
        us = np.array([0.0, 0.2, 0.5, 0.7, 0.999, 0.3], np.float32)
        x = torch.full((6, V), -3.0, dtype=dt, device=dev)
        token, _ = draw(p4q, dev, x, us, top_k=np.array(ks, np.int32))
        want = [math.floor(float(u) * ((k or V) * 2 ** 31)) // 2 ** 31 for u, k in zip(us, ks)]
        assert token.tolist() == want
        ps = np.array([0.25, 0.5, 1e-9, 0.75, 0.3, 0.999], np.float32)
        token, lp = draw(p4q, dev, x, us, top_p=ps)
        for n in range(6):
            kept = max(1, -(-max(1, math.ceil(float(ps[n]) * (V * 2 ** 31))) // 2 ** 31))
            assert token[n] == math.floor(float(us[n]) * (kept * 2 ** 31)) // 2 ** 31
            assert abs(lp[n] + math.log(kept)) < 1e-5


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("V", [900, 32003, 131071])
def test_the_largest_logits_lie_side_by_side(p4q, dev, dt, V):
    """Rising rows, a heap of large logits in one place, and rows with fewer finite logits than a top-k asks for."""
    rows = 8
    x = logits(dev, rows, V, dt, seed=11).float()
    x[0] = torch.linspace(-30, 0, V, device=dev)
    x[1] = torch.linspace(0, -9, V, device=dev)
    x[2, 300:556] = torch.linspace(11, 15, 256, device=dev)  # (seen by few of the threads that load the row)
    x[3, V - 40:] = 20.0
    x[4, :] = float("-inf")
    x[4, 100:150] = torch.linspace(0, 3, 50, device=dev)
    x[5, :] = -float("inf")
    x[5, ::97] = 1.0
    x[6, 7:] -= 500.0  # past the range of weights that are not 0
    x = x.to(dt)
    xs = x.float().cpu().numpy()
    u = np.random.default_rng(V).random(rows).astype(np.float32)
    for k in (1, 3, 40, 49, 50, 51, 130, 255, 256, 257, 600):
        ks = np.full(rows, k, np.int32)
        for params in ({"top_k": ks}, {"top_k": ks, "top_p": np.full(rows, 0.8, np.float32)},
                       {"top_k": ks, "min_p": np.full(rows, 0.02, np.float32)}):
            token, lp = draw(p4q, dev, x, u, **params)
            for n in range(rows):
                check_row(xs[n], float(u[n]), int(token[n]), float(lp[n]), **{key: val[n] for key, val in params.items()})


def test_ties_at_the_cut_go_to_the_lower_index(p4q, dev):
    """Three levels of logits, far apart in index, in no order; the cut falls inside a level."""
    V = 40000
    rng = np.random.default_rng(5)
    level = rng.integers(0, 3, V)
    x = torch.from_numpy(np.array([0.0, -1.0, -300.0], np.float32)[level]).to(dev).repeat(8, 1)
    n0, n1 = int((level == 0).sum()), int((level == 1).sum())
    ks = [1, n0 - 1, n0, n0 + 1, n0 + n1 // 2, n0 + n1, n0 + n1 + 7, 0]
    us = np.linspace(0, 1, 8, endpoint=False).astype(np.float32) + np.float32(0.0625)
    token, lp = draw(p4q, dev, x, us, top_k=np.array(ks, np.int32))
    xs = x.cpu().numpy()
    for n in range(8):
        check_row(xs[n], float(us[n]), int(token[n]), float(lp[n]), top_k=ks[n])
    # everything of level 0 and the first of level 1: the last kept token is the first -1
    u = np.full(8, 1 - 2.0 ** -24, np.float32)
    token, _ = draw(p4q, dev, x[:1], u[:1], top_k=np.array([n0], np.int32))
    assert token[0] == np.nonzero(level == 0)[0][-1]


@pytest.mark.parametrize("dt", TYPES)
def test_masked_infinite_and_nan_logits(p4q, dev, dt):
    V = 9001
    inf, nan = float("inf"), float("nan")
    low = float(torch.finfo(dt).min)
    base = logits(dev, 10, V, dt, seed=7).clone()
    base[0, :] = -inf                       # nothing
    base[1, :] = nan                        # nothing either
    base[2, :] = -inf; base[2, 4567] = -2.0  # noqa: E702  one token
    base[3, ::2] = -inf
    base[4, 1::3] = nan
    base[5, 17] = inf; base[5, 8000] = inf  # noqa: E702  two infinite ones share all
    base[6, :] = low                        # a row of the lowest value: all alike
    base[7, :] = low; base[7, 9000] = 0.0   # noqa: E702
    base[8, :5000] = low
    base[9, 1:] = -inf; base[9, 0] = low    # noqa: E702
    xs = base.float().cpu().numpy()
    u = np.array([0.5, 0.5, 0.9, 0.4, 0.6, 0.75, 0.31, 0.99, 0.01, 0.5], np.float32)
    full = {"temperature": np.full(10, 0.8, np.float32), "top_k": np.full(10, 4000, np.int32),
            "top_p": np.full(10, 0.9, np.float32), "min_p": np.full(10, 1e-4, np.float32)}
    names = {"temperature": "T", "top_k": "top_k", "top_p": "top_p", "min_p": "min_p"}
    for keys in ((), ("temperature",), ("top_k",), ("top_p",), ("min_p",), tuple(full)):
        params = {k: full[k] for k in keys}
        token, lp = draw(p4q, dev, base, u, **params)
        assert token[2] == 4567 and token[7] == 9000 and token[9] == 0 and token[0] == -1 and token[1] == -1
        for n in range(10):
            row = xs[n]
            if n == 5:
                assert token[5] == (17 if "top_p" in keys and 0.9 <= 0.5 else 8000) and abs(lp[5] + math.log(2)) < 1e-6
                continue
            check_row(row, float(u[n]), int(token[n]), float(lp[n]), **{names[k]: params[k][n] for k in keys})
    token, lp = draw(p4q, dev, base, u, temperature=np.zeros(10, np.float32))  # greedy
    want = [-1, -1] + [int(np.argmax(np.where(np.isnan(r), -np.inf, r))) for r in xs[2:]]
    assert token.tolist() == want


def test_greedy_takes_the_first_of_equal_maxima(p4q, dev):
    for V in (100, 33333):
        x = logits(dev, 4, V, torch.float16, seed=1).clone()
        for n, at in enumerate(((V - 1,), (5, V // 2), (0, V - 1), (V // 3, V // 3 + 1))):
            x[n, list(at)] = 50.0
        token, lp = draw(p4q, dev, x, np.full(4, 0.99, np.float32), temperature=np.zeros(4, np.float32))
        assert token.tolist() == [V - 1, 5, 0, V // 3] and lp.tolist() == [0.0] * 4


def test_negative_and_positive_zero_are_equal(p4q, dev):
    x = torch.full((1, 1000), -20.0, device=dev)
    x[0, 100] = 0.0
    x[0, 50] = -0.0
    token, _ = draw(p4q, dev, x, [0.9], top_k=np.array([1], np.int32))
    assert token[0] == 50


def test_the_share_of_each_token(p4q, dev):
    """Uniform numbers on a grid give each token its share of them, to within the grid."""
    V, n = 50, 20000
    x = logits(dev, 1, V, torch.float32, seed=11, spread=1.0)
    u = ((np.arange(n) + 0.5) / n).astype(np.float32)
    token, lp = draw(p4q, dev, x.expand(n, V).contiguous(), u, top_k=np.full(n, 12, np.int32))
    p = np.exp(x[0].double().cpu().numpy())
    out = np.argsort(-p)[12:]
    p[out] = 0
    p /= p.sum()
    share = np.bincount(token, minlength=V) / n
    assert np.all(np.abs(share - p) <= 1.5 / n + 1e-5)
    assert np.allclose(lp, np.log(p[token]), atol=1e-5)


@pytest.mark.parametrize("rows", [1, 2, 37, 151, 153, 400])
def test_rows_do_not_depend_on_each_other(p4q, dev, rows):
    """A row alone and among others: the same token and the same bits."""
    V = 32000
    x = logits(dev, rows, V, torch.bfloat16, seed=rows)
    rng = np.random.default_rng(rows)
    u = rng.random(rows).astype(np.float32)
    k = rng.integers(0, 400, rows).astype(np.int32)
    p = rng.uniform(0.5, 1.05, rows).astype(np.float32)
    token, lp = draw(p4q, dev, x, u, top_k=k, top_p=p)
    for n in range(0, rows, max(1, rows // 5)):
        t1, l1 = draw(p4q, dev, x[n:n + 1], u[n:n + 1], top_k=k[n:n + 1], top_p=p[n:n + 1])
        assert t1[0] == token[n] and l1[0] == lp[n]


def test_rows_at_every_alignment(p4q, dev):
    """Rows that begin at every element of 16 bytes, and the values beside them are not theirs."""
    for dt in TYPES:
        for V in (1, 5, 257, 1030):
            big = torch.full((20, V + 3), 60.0, dtype=dt, device=dev)
            x = logits(dev, 20, V, dt, seed=V)
            big[:, 2:V + 2] = x
            u = np.random.default_rng(1).random(20).astype(np.float32)
            p = np.full(20, 0.8, np.float32)
            a, la = draw(p4q, dev, big[:, 2:V + 2], u, top_p=p)
            b, lb = draw(p4q, dev, x.contiguous(), u, top_p=p)
            assert a.tolist() == b.tolist() and la.tolist() == lb.tolist()


def test_another_stream_and_a_graph(p4q, dev):
    x = logits(dev, 5, 32000, torch.float16, seed=2)
    u = torch.rand((5,), device=dev)
    p = torch.full((5,), 0.9, device=dev)
    t0, l0 = p4q.sample(x, u, top_p=p)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        t1, l1 = p4q.sample(x, u, top_p=p)
    s.synchronize()
    assert torch.equal(t0, t1) and torch.equal(l0, l1)
    t2, l2 = torch.empty_like(t0), torch.empty_like(l0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p4q.p4q_sample(x, u, t2, l2, top_p=p)
    u.copy_(u.flip(0))
    graph.replay()
    torch.cuda.synchronize()
    t3, l3 = p4q.sample(x, u, top_p=p)
    assert torch.equal(t2, t3) and torch.equal(l2, l3)


def test_the_binding_refuses(p4q, dev):
    x = torch.zeros((3, 100), device=dev)
    u = torch.zeros((3,), device=dev)
    t = torch.full((3,), -7, dtype=torch.int32, device=dev)
    for args, kw, error in [((x.double(), u, t), {}, TypeError), ((x.t(), u, t), {}, TypeError), ((x, u[:2], t), {}, ValueError),
                            ((x, u, t.long()), {}, TypeError), ((x, None, t), {}, TypeError), ((x, u, None), {}, TypeError),
                            ((x, u, t), {"top_k": u}, TypeError), ((x, u, t), {"top_p": t}, TypeError),
                            ((x, u, t), {"temperature": u[:1]}, ValueError), ((x[:, :0], u, t), {}, p4q.P4QError),
                            ((x[0], u, t), {}, TypeError)]:
        with pytest.raises(error):
            p4q.p4q_sample(*args, **kw)
    big = torch.empty((1, 262145), dtype=torch.float16, device=dev)
    with pytest.raises(p4q.P4QError):
        p4q.p4q_sample(big, u[:1], t[:1])
    torch.cuda.synchronize()
    assert t.tolist() == [-7] * 3
    p4q.p4q_sample(x[:0], u[:0], t[:0])  # nothing
