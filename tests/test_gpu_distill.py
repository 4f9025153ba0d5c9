"""Distillation (kgq_distill) against the definition in 64 bits: loss and
gradient over short and long rows, both types, shorter lists, masks, entities
that occur twice, strides, the gradient in place, graph replays."""

import numpy as np
import pytest

from paper_2503_02172_amd import kgq
from tests import rows_ref as R

pytestmark = pytest.mark.gpu


def engine(N, **kw):
    return kgq.Engine(kgq.GQE, N, 1, 4, 24.0, 1, **kw)


def inputs(B, N, K, seed):
    rng = np.random.default_rng(seed)
    z = rng.normal(8.0, 2.0, (B, N)).astype(np.float32)
    for b in range(B):
        n = int(rng.integers(0, min(N, 30) + 1))
        z[b, rng.choice(N, n, replace=False)] += rng.uniform(4, 14, n).astype(np.float32)
    t = z + rng.normal(0, 1, (B, N)).astype(np.float32)
    idx = np.argsort(-t, 1, kind="stable")[:, :K].astype(np.int32)
    return z, idx, np.take_along_axis(t, idx, 1), rng.uniform(0.1, 2.0, B).astype(np.float32)


def call(eng, z, idx, t, tau, w, dtype="f32", pad=0, out=None, **kw):
    import torch
    N = z.shape[1]
    buf = torch.full((z.shape[0], N + pad), 1e30, device="cuda")
    buf[:, :N] = torch.as_tensor(z, device="cuda")
    tz = (buf.bfloat16() if dtype == "bf16" else buf)[:, :N]
    used = tz.float().cpu().numpy()
    c = lambda a: None if a is None else torch.as_tensor(a, device="cuda")
    loss, grad = eng.distill(tz, c(idx), c(t), temperature=tau, weight=c(w), out=tz if out == "scores" else out, **kw)
    torch.cuda.synchronize()
    n = lambda a: None if a is None else a.float().cpu().numpy()
    return n(loss), n(grad), used


def check(eng, z, idx, t, tau, w, what, dtype="f32", **kw):
    loss, grad, used = call(eng, z, idx, t, tau, w, dtype, **kw)
    ww = np.ones(len(z)) if w is None else w.astype(np.float64)
    rl, rg, lb, gb = R.distill(used, idx, t, tau, ww)
    if dtype == "bf16":
        gb = gb + R.U16 * (np.abs(rg) + gb)
    for name, got, ref, bound in (("loss", loss, rl, lb), ("grad", grad, rg, gb)):
        assert np.array_equal(np.isnan(got), np.isnan(ref)), f"{what}: NaN in {name}"
        inf = np.isinf(ref)
        assert np.array_equal(got[inf], ref[inf].astype(np.float32)), f"{what}: infinite {name}"
        ok = np.isfinite(ref)
        over = np.abs(got[ok] - ref[ok]) - bound[ok]
        assert not (over > 0).any(), f"{what}: {name} off by {np.abs(got[ok] - ref[ok]).max():.3g}, over its bound by {over.max():.3g}"
    return loss, grad


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N", [1, 2, 63, 65, 1000, 4097, 14505, 63361, 65537, 140001])
def test_gpu_distill_sizes(N, dtype):
    eng = engine(N)
    for K in sorted({1, min(N, 10), min(N, 100), min(N, 1024)}):
        z, idx, t, w = inputs(3, N, K, N + K)
        for tau in (1.0, 4.0):
            print(f"[distill] N={N} K={K} {dtype} tau={tau}", flush=True)
            check(eng, z, idx, t, tau, w, f"N={N} K={K} tau={tau}", dtype=dtype)


@pytest.mark.parametrize("B,N,K", [(300, 1500, 20), (1025, 40, 5), (70, 63361, 100), (600, 17000, 30)])
def test_gpu_distill_batches(B, N, K):
    eng = engine(N)
    z, idx, t, w = inputs(B, N, K, 5)
    a = check(eng, z, idx, t, 2.0, w, "batch")
    b = check(eng, z, idx, t, 2.0, w, "batch, odd stride", pad=3)
    c = check(eng, z, idx, t, 2.0, w, "batch, in place", pad=3, out="scores")
    for x in (b, c):
        np.testing.assert_array_equal(a[0], x[0])
    again = call(eng, z, idx, t, 2.0, w)
    np.testing.assert_array_equal(a[0], again[0])
    np.testing.assert_array_equal(a[1], again[1])


@pytest.mark.parametrize("N", [70, 14505, 70000])
def test_gpu_distill_gradient_in_place_and_single_outputs(N):
    eng = engine(N)
    z, idx, t, w = inputs(4, N, 20, 6)
    loss, grad = check(eng, z, idx, t, 2.0, w, "both")
    l2, g2, _ = call(eng, z, idx, t, 2.0, w, grad=False)
    assert g2 is None
    np.testing.assert_array_equal(l2, loss)
    l3, g3, _ = call(eng, z, idx, t, 2.0, w, loss=False)
    assert l3 is None
    np.testing.assert_array_equal(g3, grad)
    _, g4, _ = call(eng, z, idx, t, 2.0, w, out="scores")
    np.testing.assert_array_equal(g4, grad)
    check(eng, z, idx, t, 2.0, None, "weight 1")
    for dtype in ("f32", "bf16"):
        check(eng, z, idx, t, 2.0, w, "in place", dtype=dtype, out="scores", pad=1)


@pytest.mark.parametrize("N", [90, 20000, 80000])
def test_gpu_distill_lists(N):
    """Shorter lists, empty ones, an entity twice and a thousand times, ids out
    of range, lists in any order."""
    rng = np.random.default_rng(N)
    eng = engine(N)
    K = 64
    z, idx, t, w = inputs(10, N, K, 7)
    for b in range(10):
        o = rng.permutation(K)
        idx[b], t[b] = idx[b, o], t[b, o]
    idx[0, 5:] = -1
    idx[1] = -1                                                # no target
    t[2] = -np.inf                                             # nothing left of it
    t[3, 1:] = -np.inf
    idx[4] = idx[4, 0]                                         # one entity
    idx[5, ::2] = idx[5, 1::2]                                 # every entity twice
    idx[6, 3], idx[6, 4] = N, -7                               # no entities
    idx[7, 0], t[7, 0] = -1, np.nan                            # left out whatever its score
    idx[8, :2], t[8, :2] = [0, N - 1], np.inf                  # infinite teacher scores share
    w[9] = 0.0
    check(eng, z, idx, t, 1.5, w, "lists")
    eng.set_checked(True)
    with pytest.raises(kgq.KgqError) as e:
        call(eng, z, idx, t, 1.5, w)
    assert e.value.name == "OUT_OF_RANGE"
    idx[6, 3:5] = -1
    check(eng, z, idx, t, 1.5, w, "lists, checked")
    big = np.resize(idx[0, :5], (10, 1024)).astype(np.int32)   # 1,024 entries of five entities
    check(eng, z, big, rng.normal(0, 1, big.shape).astype(np.float32), 1.5, w, "repeated")


@pytest.mark.parametrize("N", [90, 20000, 80000])
def test_gpu_distill_masks_and_infinities(N):
    eng = engine(N)
    z, idx, t, w = inputs(9, N, 10, 8)
    low = np.finfo(np.float32).min
    rest = np.ones(N, bool)
    rest[idx[0]] = False
    z[0, rest] = -np.inf                                       # only the list is left
    z[1, rest] = low
    z[2, idx[2, 3]] = -np.inf                                  # a listed entity masked: loss inf
    z[3] = -np.inf                                             # NaN
    z[4] = low                                                 # all equal
    z[5, 7] = np.nan
    z[6, 7] = np.inf
    t[7, 2] = np.nan
    z[8, 0], z[8, 1] = 3e38, -3e38
    idx[8, 0] = 0
    check(eng, z, idx, t, 2.0, w, "masks")
    w[:] = 0.0
    _, grad, _ = call(eng, z, idx, t, 2.0, w)
    assert (grad == 0.0).all()                                 # padding rows of any content


def test_gpu_distill_far_scores():
    """Scores far below and far from zero: the gradient keeps its relative error."""
    N = 3001
    eng = engine(N)
    rng = np.random.default_rng(9)
    z = np.stack([rng.uniform(-80, 0, N), 1e4 + rng.uniform(-40, 0, N), -1e4 + rng.uniform(-40, 0, N),
                  rng.uniform(-1e-6, 1e-6, N)]).astype(np.float32)
    idx = np.argsort(-z, 1)[:, :7].astype(np.int32)
    t = np.take_along_axis(z, idx, 1)
    for tau in (0.5, 1.0, 30.0):
        check(eng, z, idx, t, tau, None, f"far, tau {tau}")


def test_gpu_distill_gradient_against_differences():
    N = 500
    eng = engine(N)
    z, idx, t, w = inputs(3, N, 20, 10)
    _, grad, _ = call(eng, z, idx, t, 2.0, w)
    rng = np.random.default_rng(1)
    h = 1e-5
    for _ in range(4):
        v = rng.normal(0, 1, z.shape)
        up, down = (R.distill(z + s * h * v, idx, t, 2.0, w)[0] for s in (1, -1))
        d = (w * (up - down)).sum() / (2 * h)
        # the gradient's own bound is 1e-6 of it; the differences' error h^2
        assert abs(d - (grad * v).sum()) < 1e-5 * np.abs(grad * v).sum()


def test_gpu_distill_row_offsets_past_32_bits():
    import torch
    N, ld = 5000, 1_100_000_000
    eng = engine(N)
    z, idx, t, w = inputs(3, N, 10, 11)
    big = torch.empty(2 * ld + N, dtype=torch.float32, device="cuda")
    tz = torch.as_strided(big, (3, N), (ld, 1))
    tz.copy_(torch.as_tensor(z))
    c = lambda a: torch.as_tensor(a, device="cuda")
    ref = eng.distill(c(z), c(idx), c(t), weight=c(w))
    got = eng.distill(tz, c(idx), c(t), weight=c(w), out=tz)
    assert torch.equal(ref[0], got[0]) and torch.equal(ref[1], got[1])


def test_gpu_distill_captured_and_replayed():
    import torch
    c = lambda a: torch.as_tensor(a, device="cuda")
    for N in (20000, 90000):
        eng = engine(N)
        sets = [tuple(c(a) for a in inputs(5, N, 50, 20 + i)) for i in range(4)]
        z, idx, t, w = (a.clone() for a in sets[0])
        eng.distill(z, idx, t, weight=w)
        torch.cuda.synchronize()
        graphs = []
        for tau in (1.0, 3.0):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                out = eng.distill(z, idx, t, temperature=tau, weight=w)
            graphs.append((tau, g, out))
        for i in range(4):
            for dst, src in zip((z, idx, t, w), sets[i]):
                dst.copy_(src)
            for tau, g, out in graphs:
                eager = eng.distill(z, idx, t, temperature=tau, weight=w)
                g.replay()
                torch.cuda.synchronize()
                assert torch.equal(out[0], eager[0]) and torch.equal(out[1], eager[1]), (N, i, tau)


def test_gpu_distill_binding_refusals():
    import torch
    eng = engine(100)
    z = torch.zeros(4, 200, device="cuda")
    s = z[:, :100]
    idx, t = torch.zeros(4, 3, dtype=torch.int32, device="cuda"), torch.zeros(4, 3, device="cuda")
    for call_ in (lambda: eng.distill(s, idx.long(), t), lambda: eng.distill(s, idx, t.double()),
                  lambda: eng.distill(s.half(), idx, t), lambda: eng.distill(s, idx, t, weight=t[0].cpu()),
                  lambda: eng.distill(s.t().contiguous().t(), idx, t)):
        with pytest.raises(TypeError):
            call_()
    for call_ in (lambda: eng.distill(s, idx[:2], t), lambda: eng.distill(s, idx, t[:, :2].contiguous()),
                  lambda: eng.distill(z, idx, t), lambda: eng.distill(s, idx, t, out=z[:, 50:150]),
                  lambda: eng.distill(s, idx, t, out=s.bfloat16()), lambda: eng.distill(s, idx, t, weight=t[0])):
        with pytest.raises(ValueError):
            call_()
    for kw in (dict(temperature=0.0), dict(temperature=float("nan")), dict(loss=False, grad=False)):
        with pytest.raises(kgq.KgqError):
            eng.distill(s, idx, t, **kw)


@pytest.mark.parametrize("N", [4096, 16384, 16385, 65536])
def test_gpu_distill_many_bfloat16_rows(N):
    """Rows at the ends of what a workgroup holds, few and more than two to a
    compute unit."""
    eng = engine(N)
    for B in (2, 530):
        z, idx, t, w = inputs(B, N, 50, 7)
        z[0, N // 2:] = -np.inf
        a = check(eng, z, idx, t, 2.0, w, f"B={B}", dtype="bf16")
        b = check(eng, z, idx, t, 2.0, w, f"B={B}, in place", dtype="bf16", pad=5, out="scores")
        np.testing.assert_array_equal(a[0], b[0])
        np.testing.assert_array_equal(a[1], b[1])
