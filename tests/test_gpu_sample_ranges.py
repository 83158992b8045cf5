"""The draw at the ends of the temperature's and the logits' ranges, against the
definition in 64 bits (bounds as in test_gpu_sample)."""
import numpy as np
import pytest
import torch

from test_gpu_sample import check_row, draw

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
