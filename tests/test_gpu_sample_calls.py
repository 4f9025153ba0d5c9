"""Draws (kgq_sample) from rows and with settings at the ends of their ranges,
against the definition in 64 bits."""

import numpy as np
import pytest

from paper_2503_02172_amd import kgq
from tests import rows_ref as R

pytestmark = pytest.mark.gpu


def check(eng, x, u, what, dtype="float32", T=1.0, k=0, p=1.0, m=0.0):
    import torch
    t = torch.as_tensor(x, device="cuda").to(getattr(torch, dtype))
    idx, logp = (a.cpu().numpy() for a in eng.sample(t, torch.as_tensor(u, device="cuda"), temperature=T, top_k=k,
                                                     top_p=p, min_p=m))
    for b in range(len(x)):
        R.check_draws(idx[b], logp[b], t[b].float().cpu().numpy(), u[b], f"{what} row {b}", T=T, k=k, p=p, m=m)


@pytest.mark.parametrize("N", [1, 3, 500, 9000, 66000])
def test_gpu_sample_min_p_where_every_score_is_the_lowest(N):
    """Rows of the type's lowest value alone, or with -inf beside it: they
    are equal, so min-p keeps all of them."""
    eng = kgq.Engine(kgq.GQE, N, 1, 4, 24.0, 1)
    rng = np.random.default_rng(N)
    low = np.finfo(np.float32).min
    x = np.full((4, N), low, np.float32)
    x[1, 1:] = -np.inf
    x[2, rng.random(N) < 0.5] = -3.2e38                        # far above, for a temperature below 1e36
    x[3] = rng.choice(np.float32([-3e38, -3.1e38, -2.9e38]), N)
    u = rng.random((4, 9), dtype=np.float32)
    for T in (1.0, 1e-3, 1e37):
        for s in (dict(m=0.3), dict(m=1.0), dict(k=3, m=0.01), dict(p=0.7, m=0.1)):
            check(eng, x, u, f"N={N} T={T} {s}", T=T, **s)
