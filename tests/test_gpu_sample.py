"""Drawing entities from score rows (kgq_sample) against the definition in 64
bits: every setting, short and long rows, ties, masks, infinities, strides,
both types, other streams, checked mode and graph replays."""

import numpy as np
import pytest

from paper_2503_02172_amd import kgq
from tests import rows_ref as R

pytestmark = pytest.mark.gpu


def engine(N, **kw):
    return kgq.Engine(kgq.GQE, N, 1, 4, 24.0, 1, **kw)


def scores(B, N, seed, spread=2.0):
    """A wide bulk and a few answers above it."""
    rng = np.random.default_rng(seed)
    x = rng.normal(8.0, spread, (B, N)).astype(np.float32)
    for b in range(B):
        n = int(rng.integers(0, min(N, 30) + 1))
        x[b, rng.choice(N, n, replace=False)] += rng.uniform(4, 14, n).astype(np.float32)
    return x


def uniforms(B, S, seed):
    return np.random.default_rng(seed).random((B, S), dtype=np.float32)


def run(eng, x, u, dtype="f32", pad=0, **kw):
    """(idx, logp, the scores as the kernel reads them)"""
    import torch
    t = torch.zeros(x.shape[0], x.shape[1] + pad, device="cuda")
    t[:, x.shape[1]:] = 1e30                                   # outside the rows
    t[:, :x.shape[1]] = torch.as_tensor(x, device="cuda")
    t = (t.bfloat16() if dtype == "bf16" else t)[:, :x.shape[1]]
    kw = {k: torch.as_tensor(v, device="cuda") if isinstance(v, np.ndarray) else v for k, v in kw.items()}
    idx, logp = eng.sample(t, torch.as_tensor(u, device="cuda"), **kw)
    torch.cuda.synchronize()
    return idx.cpu().numpy(), None if logp is None else logp.cpu().numpy(), t.float().cpu().numpy()


def check(eng, x, u, what, T=1.0, k=0, p=1.0, m=0.0, **kw):
    idx, logp, x = run(eng, x, u, temperature=T, top_k=k, top_p=p, min_p=m, **kw)
    for b in range(x.shape[0]):
        of = lambda v: float(v[b]) if isinstance(v, np.ndarray) else v
        R.check_draws(idx[b], logp[b], x[b], u[b], f"{what} row {b}", T=of(T), k=int(of(k)), p=of(p), m=of(m))


SETTINGS = [dict(), dict(T=0.0), dict(T=0.3), dict(T=40.0), dict(k=1), dict(k=2), dict(k=50), dict(k=1500),
            dict(p=1e-6), dict(p=0.5), dict(p=0.9), dict(p=0.99999), dict(m=0.05), dict(m=1.0),
            dict(T=0.7, k=40, p=0.8), dict(T=2.0, k=1000, p=0.95, m=0.01), dict(p=0.7, m=0.2)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N", [1, 2, 63, 64, 65, 1000, 4097, 14505, 63361, 65537, 140001])
def test_gpu_sample_settings(N, dtype):
    eng = engine(N)
    B = 3
    x, u = scores(B, N, N), uniforms(B, 5, N + 1)
    for s in SETTINGS:
        print(f"[sample] N={N} {dtype} {s}", flush=True)
        check(eng, x, u, f"N={N} {s}", dtype=dtype, **s)


@pytest.mark.parametrize("N", [300, 20000])
def test_gpu_sample_rows_have_their_own_settings(N):
    rng = np.random.default_rng(N)
    B = 40
    eng = engine(N)
    x, u = scores(B, N, 7), uniforms(B, 9, 8)
    T = rng.choice([0.0, 0.5, 1.0, 3.0], B).astype(np.float32)
    k = rng.choice([0, 1, 7, 300, 5000], B).astype(np.int32)
    p = rng.choice([0.2, 0.9, 1.0, 2.0], B).astype(np.float32)
    m = rng.choice([0.0, 0.03, 0.5], B).astype(np.float32)
    check(eng, x, u, "own settings", T=T, k=k, p=p, m=m, pad=3)
    check(eng, x, u, "own top-k only", k=k)


def test_gpu_sample_settings_out_of_range_draw_nothing():
    B, N = 8, 100
    eng = engine(N)
    x, u = scores(B, N, 1), uniforms(B, 4, 2)
    T = np.array([1, -1, np.nan, np.inf, 1, 1, 1, 1], np.float32)
    k = np.array([0, 0, 0, 0, -3, 0, 0, 0], np.int32)
    p = np.array([1, 1, 1, 1, 1, 0, 1, np.nan], np.float32)
    m = np.array([0, 0, 0, 0, 0, 0, 1.5, 0], np.float32)
    kw = dict(temperature=T, top_k=k, top_p=p, min_p=m)
    idx, logp, _ = run(eng, x, u, **kw)
    assert (idx[0] >= 0).all() and (idx[1:] == -1).all() and np.isnan(logp[1:]).all()
    eng.set_checked(True)
    with pytest.raises(kgq.KgqError) as e:
        run(eng, x, u, **kw)
    assert e.value.name == "INVALID_ARG"
    run(eng, x, u)                                             # the next call starts without the last one's error


@pytest.mark.parametrize("N", [65, 5000, 70000])
def test_gpu_sample_ties(N):
    """Equal scores: cuts fall between equal entities, by index; many bins of
    one value; -0 and +0 equal."""
    eng = engine(N)
    rng = np.random.default_rng(N)
    x = np.stack([np.full(N, 3.25), rng.integers(-3, 3, N) / 4.0, np.where(np.arange(N) % 2, 0.0, -0.0),
                  np.where(np.arange(N) == N // 2, 1.0, 0.0), np.full(N, -1e30)]).astype(np.float32)
    u = uniforms(5, 7, N)
    u[:, 0], u[:, 1] = 0.0, np.float32(1) - np.float32(2.0 ** -24)
    for s in [dict(), dict(k=33), dict(k=N - 1), dict(p=0.5), dict(p=0.123, k=60), dict(m=1.0), dict(T=0.0)]:
        check(eng, x, u, f"ties {s}", **s)


@pytest.mark.parametrize("N", [200, 9000, 66000])
def test_gpu_sample_masks_and_infinities(N):
    eng = engine(N)
    x = scores(9, N, N)
    rng = np.random.default_rng(N + 5)
    low = np.finfo(np.float32).min
    x[0] = -np.inf                                             # nothing left
    x[1] = np.nan
    x[2, 1:] = -np.inf                                         # one left
    x[3, :-1] = np.nan                                         # one left, the last
    x[4, rng.random(N) < 0.9] = -np.inf
    x[5, rng.random(N) < 0.9] = low                            # masked by the type's lowest value
    x[6] = low                                                 # every one of them: all equal
    x[7, [3, N - 1]] = np.inf                                  # infinite scores share the weight
    x[8, 5], x[8, 6] = 3e38, -3e38
    u = uniforms(9, 6, 3)
    for s in [dict(), dict(k=20), dict(k=N // 2), dict(p=0.9), dict(T=0.5, k=100, p=0.9, m=0.1), dict(T=0.0)]:
        print(f"[masks] N={N} {s}", flush=True)
        check(eng, x, u, f"masks {s}", **s)


@pytest.mark.parametrize("spread", [0.0, 1e-6, 1e-3, 300.0, 1e6])
def test_gpu_sample_flat_and_steep_rows(spread):
    N = 30000
    eng = engine(N)
    rng = np.random.default_rng(11)
    x = (5.0 + spread * rng.normal(0, 1, (3, N))).astype(np.float32)
    x[2] = np.where(rng.random(N) < 0.5, x[2], (5.0 - spread * 2.0 ** -(np.arange(N) % 100)).astype(np.float32))
    u = uniforms(3, 5, 12)
    for s in [dict(), dict(k=5000), dict(k=29999), dict(p=0.3), dict(p=0.97), dict(T=1e-3, p=0.9), dict(k=300, p=0.5)]:
        check(eng, x, u, f"spread {spread} {s}", **s)


def test_gpu_sample_random_numbers_outside():
    N = 500
    eng = engine(N)
    x = scores(1, N, 4)
    x[0, -3:] = -np.inf
    u = np.array([[0.0, 1.0, 2.0, -1.0, np.nan, np.inf, -np.inf, 0.5]], np.float32)
    for s in [dict(), dict(k=9)]:
        idx, _, _ = run(eng, x, u, temperature=1.0, top_k=s.get("k", 0))
        w, _ = R.kept(x[0], **s)
        first, last = np.nonzero(w)[0][[0, -1]]
        assert idx[0].tolist()[:7] == [first, last, last, first, first, last, first]


@pytest.mark.parametrize("B,N,S", [(1, 7, 1), (300, 800, 1), (2, 3000, 1000), (1025, 37, 2)])
def test_gpu_sample_batches_and_draws(B, N, S):
    eng = engine(N)
    x, u = scores(B, N, 21), uniforms(B, S, 22)
    check(eng, x, u, "batch", T=1.3, p=0.95, pad=5)
    idx, logp, _ = run(eng, x, u, temperature=1.3, top_p=0.95, pad=5, logp=False)
    assert logp is None
    again, _, _ = run(eng, x, u, temperature=1.3, top_p=0.95, pad=5)
    np.testing.assert_array_equal(idx, again)


def test_gpu_sample_shares_follow_the_weights():
    """Evenly spaced numbers: every entity is drawn in proportion, within one."""
    N, S = 60, 4096
    eng = engine(N)
    x = scores(1, N, 31)
    u = ((np.arange(S) + 0.5) / S).astype(np.float32)[None]
    idx, _, _ = run(eng, x, u, temperature=4.0)
    w = R.weights(x[0], 4.0)
    assert np.abs(np.bincount(idx[0], minlength=N) - S * w / w.sum()).max() <= 1.0


def test_gpu_sample_row_offsets_past_32_bits():
    import torch
    N, ld = 5000, 1_100_000_000
    eng = engine(N)
    big = torch.empty(2 * ld + N, dtype=torch.float32, device="cuda")
    t = torch.as_strided(big, (3, N), (ld, 1))
    x, u = scores(3, N, 41), uniforms(3, 4, 42)
    t.copy_(torch.as_tensor(x))
    idx, logp = eng.sample(t, torch.as_tensor(u, device="cuda"), top_p=0.9)
    idx, logp = idx.cpu().numpy(), logp.cpu().numpy()
    for b in range(3):
        R.check_draws(idx[b], logp[b], x[b], u[b], f"row {b}", p=0.9)


def test_gpu_sample_on_another_stream():
    import torch
    N = 6000
    eng = engine(N)
    x, u = scores(4, N, 51), uniforms(4, 4, 52)
    s = torch.cuda.Stream()
    tx, tu = torch.as_tensor(x, device="cuda"), torch.as_tensor(u, device="cuda")
    s.wait_stream(torch.cuda.current_stream())
    for stream in (s, s.cuda_stream):
        idx, logp = eng.sample(tx, tu, top_k=30, stream=stream)
        s.synchronize()
        for b in range(4):
            R.check_draws(idx[b].cpu().numpy(), logp[b].cpu().numpy(), x[b], u[b], f"row {b}", k=30)


def test_gpu_sample_captured_and_replayed():
    """Two captured graphs and eager calls between their replays; every replay
    reads what its inputs hold then."""
    import torch
    N = 20000
    eng = engine(N)
    u = uniforms(6, 8, 61)
    tx = [torch.as_tensor(scores(6, N, 62 + i), device="cuda") for i in range(2)]
    tu = torch.as_tensor(u, device="cuda")
    kw = [dict(top_p=0.9), dict(top_k=64, min_p=0.01)]
    eng.sample(tx[0], tu)
    torch.cuda.synchronize()
    graphs = []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = eng.sample(tx[i], tu, **kw[i])
        graphs.append((g, out))
    for turn in range(3):
        for i, (g, out) in enumerate(graphs):
            tx[i].copy_(torch.as_tensor(scores(6, N, 70 + 10 * turn + i)))
            eager = eng.sample(tx[i], tu, **kw[i])
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out[0], eager[0]) and torch.equal(out[1], eager[1]), (turn, i)
    eng.set_checked(True)
    g = torch.cuda.CUDAGraph()
    with pytest.raises(kgq.KgqError), torch.cuda.graph(g):
        eng.sample(tx[0], tu)


def test_gpu_sample_binding_refusals():
    import torch
    eng = engine(100)
    x, u = torch.zeros(2, 100, device="cuda"), torch.zeros(2, 3, device="cuda")
    one = torch.ones(2, device="cuda")
    for call in (lambda: eng.sample(x.t(), u), lambda: eng.sample(x, u.double()), lambda: eng.sample(x.half(), u),
                 lambda: eng.sample(x, u, top_k=one), lambda: eng.sample(x, u, temperature=one.cpu())):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: eng.sample(x[:, :99], u), lambda: eng.sample(x, u[:1]), lambda: eng.sample(x, u[0]),
                 lambda: eng.sample(x, u, temperature=one[:1])):
        with pytest.raises(ValueError):
            call()
    for kw in (dict(temperature=-1.0), dict(top_k=-1), dict(top_p=0.0), dict(min_p=2.0)):
        with pytest.raises(kgq.KgqError):
            eng.sample(x, u, **kw)
    with pytest.raises(kgq.KgqError):
        eng.sample(x, u[:, :0].contiguous())
    with pytest.raises(kgq.KgqError):
        eng.sample(x.expand(2, 100)[:1].expand(2, 100), u)     # a row stride of 0


@pytest.mark.parametrize("N", [262145, 327680, 327681, 500009])
def test_gpu_sample_long_rows(N):
    """Rows beyond what the running sums hold at 64 scores each, and beyond
    those that are drawn from in pieces; with ties, which the first search
    does not resolve."""
    eng = engine(N)
    x, u = scores(2, N, N), uniforms(2, 5, N + 1)
    x[1] = np.random.default_rng(N).integers(-3, 3, N) / 4.0
    for s in [dict(), dict(T=0.0), dict(k=50), dict(k=N - 1), dict(p=0.9), dict(m=0.05), dict(T=2.0, k=5000, p=0.95)]:
        print(f"[sample] N={N} {s}", flush=True)
        check(eng, x, u, f"N={N} {s}", **s)


@pytest.mark.parametrize("N", [300, 70000])
def test_gpu_sample_more_draws_than_are_taken_together(N):
    eng = engine(N)
    x, u = scores(2, N, 5), uniforms(2, 2500, 6)
    for s in [dict(), dict(p=0.8), dict(k=20)]:
        check(eng, x, u, f"N={N} {s}", **s)


def test_gpu_sample_calls_that_overlap():
    """Calls on four streams at once, each with its own workspace, give what
    they give alone; one handle in checked mode among them."""
    import torch
    N, B = 30011, 40
    eng, checked = engine(N), engine(N)
    checked.set_checked(True)
    streams = [torch.cuda.Stream() for _ in range(4)]
    u = torch.as_tensor(uniforms(B, 16, 1), device="cuda")
    args = [(e, torch.as_tensor(scores(B, N, 80 + i), device="cuda"), kw) for i, (e, kw) in
            enumerate(((eng, dict()), (eng, dict(top_p=0.9)), (checked, dict()), (eng, dict(top_k=77))))]
    alone = [e.sample(t, u, **kw) for e, t, kw in args]
    torch.cuda.synchronize()
    outs = [[e.sample(t, u, stream=s, **kw) for s, (e, t, kw) in zip(streams, args)] for _ in range(5)]
    torch.cuda.synchronize()
    for turn in outs:
        for got, want in zip(turn, alone):
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("N", [4096, 4097, 9001, 16384, 16385, 65536])
def test_gpu_sample_few_and_many_rows(N):
    """Rows at the ends of what a workgroup holds, few and more than one to a
    compute unit."""
    eng = engine(N)
    for B in (2, 259):
        x, u = scores(B, N, N + B), uniforms(B, 3, N)
        x[0] = np.random.default_rng(N).integers(-3, 3, N) / 4.0
        x[1, N // 2:] = -np.inf
        for s in [dict(), dict(k=50), dict(p=0.9), dict(T=2.0, k=1000, p=0.95, m=0.01)]:
            check(eng, x, u, f"N={N} B={B} {s}", **s)
