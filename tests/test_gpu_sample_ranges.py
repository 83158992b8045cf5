"""The draw at the ends of the temperature's and the logits' ranges, against the
definition in 64 bits (bounds as in test_gpu_sample)."""
import numpy as np
import pytest
import torch

from test_gpu_sample import check_row, draw, logits, reference, slack

pytestmark = pytest.mark.gpu

MODES = [{}, {"top_k": 5}, {"top_k": 300}, {"top_p": 0.9}, {"top_p": 0.999}, {"min_p": 0.05}, {"min_p": 1e-6},
         {"top_k": 40, "top_p": 0.8, "min_p": 0.01}]


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T", [1e-30, 1e-36, 1e-37, 2e-38, 5e-39])
def test_logits_as_small_as_the_temperature(p4q, dev, dt, T):
    """Differences of a few T, however small T is: the weights are those of d = (x_max - x) / T."""
    V, rows = 2003, len(MODES)
    T = np.float32(T)
    rng = np.random.default_rng(7)
    d = rng.exponential(3.0, (rows, V))
    x = torch.from_numpy((-d * float(T)).astype(np.float32)).to(dt)
    xs = x.float().numpy()
    u = rng.random(rows).astype(np.float32)
    token, lp = draw(p4q, dev, x.to(dev), u, temperature=np.full(rows, T, np.float32),
                     top_k=np.array([m.get("top_k", 0) for m in MODES], np.int32),
                     top_p=np.array([m.get("top_p", 1.0) for m in MODES], np.float32),
                     min_p=np.array([m.get("min_p", 0.0) for m in MODES], np.float32))
    for n, m in enumerate(MODES):
        m = {k: (v if k == "top_k" else float(np.float32(v))) for k, v in m.items()}
        check_row(xs[n], float(u[n]), int(token[n]), float(lp[n]), T=float(T), **m)


def check_logprob(x, u, token, logprob, T=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """The logarithm is that of the token's share of some cut that the weights' errors allow
    (there may be several where a sum lies near its share) and whose interval of the token holds u."""
    x = x.astype(np.float64)
    order, e, d = reference(x, T, top_k, top_p, min_p)
    sl = slack(e, d)
    k = top_k if 0 < top_k < x.size else x.size
    order = order[:k]
    es, ss = e[order], sl[order]
    lo = hi = k
    if top_p < 1:
        mass, off = np.cumsum(es), 2 * ss.sum() + 2.0 ** -30
        need = top_p * mass[-1]
        lo, hi = (min(k, int(np.searchsorted(mass, need + s * off)) + 1) for s in (-1, 1))
    if min_p > 0:
        lo, hi = min(lo, int(np.sum(es - ss >= min_p))), min(hi, int(np.sum(es + ss >= min_p)))
    lo = max(1, min(lo, hi))
    assert hi - lo < 200, "the case says too little"
    nearest = np.inf
    for n in range(lo, hi + 1):
        kept = np.sort(order[:n])
        at = int(np.searchsorted(kept, token))
        if at == n or kept[at] != token:
            continue
        c = np.cumsum(e[kept])
        total, off = c[-1], 2 * sl[kept].sum() + 2.0 ** -30
        if not (c[at] - e[token] - off) / total <= u <= (c[at] + off) / total:
            continue
        want = -d[token] - np.log(total)
        bound = (3 * d[token] + 4) * 2.0 ** -24 + off / total + 2.0 ** -22 * (1 + abs(want))
        nearest = min(nearest, abs(logprob - want) / bound)
    assert nearest <= 1, f"{nearest} of the bound at the nearest cut of {lo} .. {hi}"


@pytest.mark.parametrize("dt", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("V", [700, 32000, 131071])
@pytest.mark.parametrize("spread", [0.3, 1.0, 4.0])
def test_logprobs_of_every_cut(p4q, dev, dt, V, spread):
    """Also where a cut lies as near a sum as the weights' errors."""
    rows = 24
    x = logits(dev, rows, V, dt, seed=V, spread=spread)
    xs = x.float().cpu().numpy()
    rng = np.random.default_rng(V)
    u = rng.random(rows).astype(np.float32)
    T = rng.uniform(0.5, 1.5, rows).astype(np.float32)
    k = rng.integers(1, 400, rows).astype(np.int32)
    p = rng.uniform(0.1, 0.98, rows).astype(np.float32)
    m = rng.uniform(0.01, 0.3, rows).astype(np.float32)
    for params in ({}, {"top_p": p}, {"temperature": T, "top_p": p}, {"top_k": k, "top_p": p}, {"top_k": k},
                   {"min_p": m}, {"top_p": p, "min_p": m}):
        token, lp = draw(p4q, dev, x, u, **params)
        for n in range(rows):
            one = {key: float(params[src][n]) if key != "top_k" else int(params[src][n])
                   for key, src in (("T", "temperature"), ("top_k", "top_k"), ("top_p", "top_p"), ("min_p", "min_p"))
                   if src in params}
            check_logprob(xs[n], float(u[n]), int(token[n]), float(lp[n]), **one)
