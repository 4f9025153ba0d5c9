"""Calls that the documentation of drawing, distillation and embedding rows
allows beyond the plain ones: gradients in layouts that have to be copied, on
streams of the caller's; a score matrix and its gradient in one buffer.
And gradients whose sums are exact, so that a token left out shows."""

import numpy as np
import pytest

from paper_2503_02172_amd import kgq

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def eng():
    e = kgq.Engine(kgq.GQE, 16, 1, 4, 24.0, 1)
    yield e
    e.close()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("n", [40, 400])
def test_gpu_embed_grad_copies_on_the_callers_stream(eng, n, dtype):
    """Gradients whose rows have no common stride, on a stream of the
    caller's, while the current stream is busy: the sums are those of the
    gradient, whatever the current stream is at. Whole numbers, so that sums
    are exact in any order."""
    import torch
    rng = np.random.default_rng(n)
    T, V, d = 9, 50, 24
    ids = torch.as_tensor(rng.integers(-1, V, (T, n)).astype(np.int32), device="cuda")
    whole = torch.as_tensor(rng.integers(-8, 9, (T, n + 1, d)), device="cuda").to(getattr(torch, dtype))
    turned = whole.transpose(0, 1).contiguous().transpose(0, 1)
    a = torch.randn(4096, 4096, device="cuda")
    s = torch.cuda.Stream()
    for layout, g in (("rows cut off", whole[:, 1:]), ("transposed", turned[:, :-1]), ("flat", whole[:, 1:].contiguous())):
        want = np.zeros((V + 1, d))
        np.add.at(want, ids.cpu().numpy().ravel(), g.double().cpu().numpy().reshape(-1, d))
        for stream in (s, s.cuda_stream, None):
            torch.cuda.synchronize()
            s.wait_stream(torch.cuda.current_stream())
            for _ in range(20):
                a = (a @ a).clamp_(-1, 1)                      # (what the copy must not wait for)
            got = eng.embed_grad(g, ids, V, stream=stream)
            torch.cuda.synchronize()
            assert np.array_equal(got.double().cpu().numpy(), want[:V]), (layout, stream)


@pytest.mark.parametrize("N", [70, 14505, 70001])
def test_gpu_distill_gradient_beside_the_scores(N):
    """Scores and their gradient as two column ranges of one buffer."""
    import torch
    B = 5
    eng = kgq.Engine(kgq.GQE, N, 1, 4, 24.0, 1)
    buf = torch.full((B, 2 * N + 3), 7.0, device="cuda")
    z, out = buf[:, 1:N + 1], buf[:, N + 1:2 * N + 1]
    z.normal_()
    t, idx = torch.randn(B, N, device="cuda").topk(20, 1)
    idx, t = idx.int(), t.contiguous()
    loss, grad = eng.distill(z.contiguous(), idx, t, temperature=2.0)
    old = z.clone()
    got = eng.distill(z, idx, t, temperature=2.0, out=out)
    assert got[1] is out and torch.equal(got[0], loss) and torch.equal(out, grad)
    assert torch.equal(z, old) and (buf[:, 0] == 7.0).all() and (buf[:, 2 * N + 1:] == 7.0).all()


def odd_rows(n, d, seed):
    """Odd numbers from -7 to 7: every sum of up to 2^21 of them is exact in
    float32 in any order, and a row left out or added twice changes it."""
    return 2.0 * np.random.default_rng(seed).integers(-4, 4, (n, d)) + 1.0


@pytest.mark.parametrize("src", ["float32", "bfloat16"])
@pytest.mark.parametrize("n,d", [(9, 3), (10, 300), (513, 1100), (2047, 8), (2048, 300), (2049, 8), (4097, 300),
                                 (9000, 6), (33333, 1100), (100000, 3), (262143, 40)])
def test_gpu_embed_grad_of_hot_ids_is_exact(eng, n, d, src):
    """Ids with most of the tokens, alone and between others, in one run or
    several, written and accumulated: every token counts once."""
    import torch
    V = 300
    g = odd_rows(n, d, n)
    tg = torch.as_tensor(g, device="cuda").to(getattr(torch, src))
    rng = np.random.default_rng(n + 1)
    at = np.arange(n)
    kinds = {"one": np.full(n, V // 2), "last": np.full(n, V - 1), "two": at % 2 * 7,
             "three quarters": np.where(at % 4 == 0, rng.integers(-1, V, n), 17), "halves": np.where(at < n // 2, 3, 4),
             "all but one": np.where(at == n // 3, 200, 100), "runs": at // 2500 % V,
             "padding between": np.where(at % 5 == 0, -1, 299)}
    for kind, ids in kinds.items():
        ti = torch.as_tensor(ids.astype(np.int32), device="cuda")
        want = np.zeros((V + 1, d))
        np.add.at(want, ids, g)
        got = eng.embed_grad(tg, ti, V, scale=0.5)
        assert np.array_equal(got.double().cpu().numpy(), 0.5 * want[:V]), kind
        old = torch.as_tensor(rng.integers(-9, 9, (V, d)), device="cuda").float()
        acc = eng.embed_grad(tg, ti, V, scale=-2.0, out=old.clone(), accumulate=True)
        assert np.array_equal(acc.double().cpu().numpy(), old.double().cpu().numpy() - 2.0 * want[:V]), kind


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("N", [300, 20001, 66001])
def test_gpu_distill_weights_at_the_end_of_float32(N, dtype):
    """A weight times the temperature up to float32's largest value gives the
    gradient, with zeros where entities are masked; one beyond it, an infinite
    one or a NaN makes the row's gradient NaN; a row without a target or of
    weight 0 has none."""
    import torch
    eng = kgq.Engine(kgq.GQE, N, 1, 4, 24.0, 1)
    rng = np.random.default_rng(N)
    B = 8
    z = rng.normal(0, 1, (B, N)).astype(np.float32)
    z[:, 5::3] = -np.inf
    idx = np.tile(np.int32([0, 1, 3]), (B, 1))
    t = rng.normal(0, 1, (B, 3)).astype(np.float32)
    idx[6] = -1
    w = np.float32([1.0, 1.6e38, -1.6e38, 3e38, np.inf, np.nan, np.inf, 0.0])
    c = lambda a: torch.as_tensor(a, device="cuda")
    tz = c(z).to(getattr(torch, dtype))
    loss, grad = eng.distill(tz, c(idx), c(t), temperature=2.0, weight=c(w))
    plain = eng.distill(tz, c(idx), c(t), temperature=2.0)
    assert torch.equal(loss, plain[0])
    assert grad[3:6].isnan().all() and not grad[6:].any()
    one = eng.distill(tz[1:3].float(), c(idx[1:3]), c(t[1:3]), temperature=2.0)[1].double()
    for row in (1, 2):
        assert torch.isfinite(grad[row]).all() and not grad[row, 5::3].any()
        want = one[row - 1] * float(w[row])
        # float32's weight-1 gradient and this one, each with 4 roundings of 2^-24 or less, then bfloat16's
        tol = 2.0 ** -21 + (2.0 ** -8 if dtype == "bfloat16" else 0.0)
        listed = torch.zeros(N, dtype=torch.bool, device="cuda")
        listed[c(idx[1]).long()] = True
        assert ((grad[row].double() - want).abs() <= tol * want.abs())[~listed].all()
        # (a listed entity's is a difference of two shares, each at most 1)
        assert ((grad[row].double() - want).abs() <= tol * want.abs() + 2.0 ** -21 * 2 * 1.6e38)[listed].all()


def test_gpu_embed_grad_copies_in_a_captured_graph(eng):
    """A gradient that has to be copied, captured: every replay copies what it
    holds then."""
    import torch
    V, T, n, d = 70, 6, 500, 20
    base = torch.zeros(n, T, d, device="cuda")
    ids = torch.zeros(T, n, dtype=torch.int32, device="cuda")
    grad = base.transpose(0, 1)
    eng.embed_grad(grad, ids, V)
    torch.cuda.synchronize()
    gr = torch.cuda.CUDAGraph()
    with torch.cuda.graph(gr):
        out = eng.embed_grad(grad, ids, V)
    for turn in range(3):
        base.copy_(torch.as_tensor(odd_rows(n * T, d, turn).reshape(n, T, d)))
        ids.copy_(torch.as_tensor(np.random.default_rng(turn).integers(-1, V, (T, n)).astype(np.int32)))
        eager = eng.embed_grad(grad, ids, V)
        gr.replay()
        torch.cuda.synchronize()
        want = np.zeros((V + 1, d))
        np.add.at(want, ids.cpu().numpy().ravel(), grad.double().cpu().numpy().reshape(-1, d))
        assert torch.equal(out, eager) and np.array_equal(out.double().cpu().numpy(), want[:V]), turn


def test_gpu_largest_counts(eng):
    """2^20 rows of scores, tables of 2^31 - 1 rows, and 2^31 - 1 tokens."""
    import torch
    if torch.cuda.mem_get_info()[0] < 90e9:
        pytest.skip("needs 60 GB of device memory")
    B, N = 1 << 20, 37
    scorer = kgq.Engine(kgq.GQE, N, 1, 4, 24.0, 1)
    x, u = torch.randn(B, N, device="cuda"), torch.rand(B, 1, device="cuda")
    idx, score = torch.randint(0, N, (B, 2), device="cuda", dtype=torch.int32), torch.randn(B, 2, device="cuda")
    some = torch.randint(0, B, (200,), device="cuda")
    some[0] = B - 1
    for kw in (dict(), dict(top_p=0.8)):
        assert torch.equal(scorer.sample(x, u, **kw)[0][some], scorer.sample(x[some], u[some], **kw)[0])
    for a, b in zip(scorer.distill(x, idx, score), scorer.distill(x[some], idx[some], score[some])):
        assert torch.equal(a[some], b)

    V = (1 << 31) - 1
    out = torch.empty(V, 1, device="cuda", dtype=torch.bfloat16)
    for n in (100, 2048, 5000):
        print(f"[counts] {V} rows, {n} tokens", flush=True)
        ids = torch.randint(0, V, (n,), device="cuda", dtype=torch.int32)
        ids[:4] = torch.tensor([V - 1, 0, -1, V - 1], dtype=torch.int32)
        out.fill_(3.0)
        eng.embed_grad(torch.ones(n, 1, device="cuda"), ids, V, out=out)
        used = sum(int((out[i:i + (1 << 28)] != 0).sum()) for i in range(0, V, 1 << 28))
        assert used == ids[ids >= 0].unique().numel() and out[V - 1, 0] == 2
        got = eng.embed(out, ids, dtype=torch.float32)
        assert got[0, 0] == 2 and got[2, 0] == 0
    del out
    torch.cuda.empty_cache()

    n, V = (1 << 31) - 1, 1 << 20
    print(f"[counts] {n} tokens", flush=True)
    ids = torch.arange(n, device="cuda", dtype=torch.int32).bitwise_and_(V - 1)
    got = eng.embed_grad(torch.ones(n, 1, device="cuda", dtype=torch.bfloat16), ids, V)
    assert (got[:-1] == 2048).all() and got[-1] == 2047
    torch.cuda.empty_cache()
    t = torch.arange(V, device="cuda").remainder_(256).bfloat16()[:, None]
    rows = eng.embed(t, ids)
    for at in range(0, n, 1 << 28):
        assert torch.equal(rows[at:at + V], t)
    assert rows[n - 1, 0] == (n - 1) % 256
    del ids, rows, got
    torch.cuda.empty_cache()
