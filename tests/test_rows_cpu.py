"""Refusals of drawing, distillation and embedding rows on a validation-only
handle (no GPU), and the definitions that the GPU tests compare with."""

import ctypes

import numpy as np
import pytest

from paper_2503_02172_amd import kgq
from tests import rows_ref as R

P = ctypes.c_void_p(4096)          # never dereferenced by a validation-only handle
OK_HOW = dict(temperature=1.0, top_k=0, top_p=1.0, min_p=0.0)


@pytest.fixture(scope="module")
def eng():
    return kgq.Engine(kgq.GQE, 50, 6, 8, 12.0, 4, device=-1)


def sample(e, batch=2, scores=P, dtype=0, ld=50, u=P, S=3, idx=P, logp=None, how=True, ws=P,
           ws_bytes=1 << 30, **kw):
    h = kgq.Sampling(**{**OK_HOW, **kw})
    return kgq.lib().kgq_sample(e.h if e else None, batch, scores, dtype, ld, ctypes.byref(h) if how else None, u, S,
                                idx, logp, ws, ws_bytes, None)


def test_sample_refusals(eng):
    assert sample(eng) == -5                                   # everything valid: no device
    assert sample(None) == -1
    for bad in (dict(batch=0), dict(batch=(1 << 20) + 1), dict(scores=None), dict(dtype=2), dict(ld=49), dict(u=None),
                dict(S=0), dict(idx=None), dict(how=False), dict(temperature=-1.0), dict(temperature=float("nan")),
                dict(temperature=float("inf")), dict(top_k=-1), dict(top_p=0.0), dict(top_p=-0.5),
                dict(top_p=float("nan")), dict(min_p=-0.1), dict(min_p=1.5), dict(min_p=float("nan"))):
        assert sample(eng, **bad) == -1, bad
    need = ctypes.c_size_t()
    L = kgq.lib()
    assert L.kgq_sample_workspace(eng.h, 2, ctypes.byref(need)) == 0 and need.value > 0
    for bad in (dict(ws=None), dict(ws=ctypes.c_void_p(4104)), dict(ws_bytes=need.value - 1)):
        assert sample(eng, **bad) == -1, bad
    assert sample(eng, ws_bytes=need.value) == -5
    for bad in (0, (1 << 20) + 1):
        assert L.kgq_sample_workspace(eng.h, bad, ctypes.byref(need)) == -1
    assert L.kgq_sample_workspace(eng.h, 2, None) == -1 and L.kgq_sample_workspace(None, 2, ctypes.byref(need)) == -1
    # a row's own settings take the place of the number, which is not looked at
    assert sample(eng, temperature=-1.0, temperature_rows=4096) == -5
    assert sample(eng, temperature=0.0, top_k=0, top_p=7.0, min_p=1.0) == -5


def distill(e, batch=2, scores=P, dtype=0, ld=50, k=5, idx=P, score=P, tau=1.0, weight=None, loss=P, grad=P, ldg=50):
    return kgq.lib().kgq_distill(e.h if e else None, batch, scores, dtype, ld, k, idx, score, tau, weight, loss, grad,
                                 ldg, None)


def test_distill_refusals(eng):
    assert distill(eng) == -5 and distill(eng, grad=None, ldg=0) == -5 and distill(eng, loss=None) == -5
    assert distill(None) == -1
    for bad in (dict(batch=0), dict(scores=None), dict(dtype=-1), dict(ld=49), dict(ldg=49), dict(k=0), dict(k=1025),
                dict(idx=None), dict(score=None), dict(tau=0.0), dict(tau=-1.0), dict(tau=float("nan")), dict(tau=1e-31),
                dict(tau=float("inf")), dict(loss=None, grad=None)):
        assert distill(eng, **bad) == -1, bad


def embed(e, table=P, dtype=0, rows=10, dim=8, ld=8, ids=P, n=4, out=P, odt=0, ldo=8):
    return kgq.lib().kgq_embed(e.h if e else None, table, dtype, rows, dim, ld, ids, n, 1.0, out, odt, ldo, None)


def test_embed_refusals(eng):
    assert embed(eng) == -5 and embed(eng, n=0, ids=None, out=None) == -5
    assert embed(None) == -1
    for bad in (dict(table=None), dict(dtype=2), dict(odt=2), dict(rows=0), dict(rows=1 << 31), dict(dim=0),
                dict(ld=7), dict(ldo=7), dict(ids=None), dict(out=None), dict(n=-1)):
        assert embed(eng, **bad) == -1, bad


def embed_grad(e, grad=P, dtype=0, n=4, dim=8, ld=8, ids=P, rows=10, out=P, odt=0, ldo=8, ws=P, ws_bytes=1 << 30):
    return kgq.lib().kgq_embed_grad(e.h if e else None, grad, dtype, n, dim, ld, ids, rows, 1.0, out, odt, ldo, 0, ws,
                                    ws_bytes, None)


def test_embed_grad_refusals(eng):
    need = ctypes.c_size_t()
    L = kgq.lib()
    assert L.kgq_embed_grad_workspace(eng.h, 10, 8, 4, ctypes.byref(need)) == 0 and need.value > 0
    for bad in ((0, 8, 4), (1 << 31, 8, 4), (10, 0, 4), (10, 8, -1)):
        assert L.kgq_embed_grad_workspace(eng.h, *bad, ctypes.byref(need)) == -1, bad
    assert L.kgq_embed_grad_workspace(eng.h, 10, 8, 4, None) == -1
    assert L.kgq_embed_grad_workspace(None, 10, 8, 4, ctypes.byref(need)) == -1
    assert L.kgq_embed_grad_workspace(eng.h, 10, 8, 4, ctypes.byref(need)) == 0
    assert embed_grad(eng, ws_bytes=need.value) == -5 and embed_grad(eng, n=0, ids=None, grad=None) == -5
    assert embed_grad(None) == -1
    for bad in (dict(grad=None), dict(dtype=2), dict(odt=-1), dict(rows=0), dict(rows=1 << 31), dict(dim=0),
                dict(ld=7), dict(ldo=7), dict(ids=None), dict(out=None), dict(n=-1), dict(ws=None),
                dict(ws=ctypes.c_void_p(4100)), dict(ws_bytes=need.value - 1)):
        assert embed_grad(eng, **bad) == -1, bad


def test_binding_refuses_host_tensors(eng):
    """What is not on the GPU, or of another type, never reaches the library."""
    import torch
    s, u = torch.zeros(2, 50), torch.zeros(2, 3)
    ids = torch.zeros(2, 4, dtype=torch.int32)
    for call in (lambda: eng.sample(s, u), lambda: eng.sample(s.double(), u), lambda: eng.distill(s, ids, u),
                 lambda: eng.embed(s, ids), lambda: eng.embed_grad(s, ids, 10)):
        with pytest.raises(TypeError):
            call()


# ---- the definitions ---------------------------------------------------------

def test_kept_by_hand():
    x = np.log([1.0, 4.0, 2.0, 4.0, 1.0])                       # weights 1/4, 1, 1/2, 1, 1/4
    np.testing.assert_allclose(R.kept(x)[0], [0.25, 1, 0.5, 1, 0.25])
    np.testing.assert_allclose(R.kept(x, k=1)[0], [0, 1, 0, 0, 0])              # ties: the lower index
    np.testing.assert_allclose(R.kept(x, k=3)[0], [0, 1, 0.5, 1, 0])
    np.testing.assert_allclose(R.kept(x, p=0.3)[0], [0, 1, 0, 0, 0])            # 1/3 of the weight
    np.testing.assert_allclose(R.kept(x, p=0.4)[0], [0, 1, 0, 1, 0])
    np.testing.assert_allclose(R.kept(x, k=3, p=0.9)[0], [0, 1, 0.5, 1, 0])     # 2 of 2.5 are short of 0.9
    np.testing.assert_allclose(R.kept(x, m=0.5)[0], [0, 1, 0.5, 1, 0], atol=0)
    np.testing.assert_allclose(R.kept(x, T=0.0)[0], [0, 1, 0, 0, 0])
    np.testing.assert_allclose(R.kept(x, T=0.5)[0], [1 / 16, 1, 0.25, 1, 1 / 16])
    assert R.kept(np.full(3, -np.inf))[0] is None and R.kept(np.array([np.nan]))[0] is None
    np.testing.assert_allclose(R.kept(np.array([np.inf, 3.0, np.inf]))[0], [1, 0, 1])


def test_distill_gradient_is_the_differences():
    rng = np.random.default_rng(3)
    z = rng.normal(0, 2, (3, 40))
    idx = np.array([[3, 7, 3, 39], [0, -1, 5, 6], [1, 2, 3, 4]])          # an entity twice, a shorter list
    t = rng.normal(0, 2, (3, 4))
    w, tau = np.array([1.0, 0.5, 2.0]), 1.7
    _, g, _, _ = R.distill(z, idx, t, tau, w)
    v = rng.normal(0, 1, z.shape)
    h = 1e-6
    up, down = (R.distill(z + s * h * v, idx, t, tau, w)[0] for s in (1, -1))
    np.testing.assert_allclose((w * (up - down)).sum() / (2 * h), (g * v).sum(), rtol=1e-7)


def test_row_widths_have_a_limit(eng):
    """2^24 columns pass every check (and end at the missing device), one more
    does not."""
    need = ctypes.c_size_t()
    n = 1 << 24
    for d, want in ((n, -5), (n + 1, -1)):
        assert embed(eng, dim=d, ld=d, ldo=d) == want
        assert kgq.lib().kgq_embed_grad_workspace(eng.h, 10, d, 4, ctypes.byref(need)) == (0 if want == -5 else -1)
        assert embed_grad(eng, dim=d, ld=d, ldo=d, ws_bytes=need.value) == want
