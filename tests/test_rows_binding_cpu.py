"""What the binding does around the calls on the caller's own arrays (draws,
distillation, embedding rows), on a validation-only handle: the checks of type
and device are switched off, so that host tensors take the way of device ones
up to the library, which ends at the missing device."""

import contextlib

import pytest
import torch

from paper_2503_02172_amd import kgq

COPIES = ("clone", "copy_", "_to_copy")


@pytest.fixture
def eng(monkeypatch):
    monkeypatch.setattr(kgq.Engine, "_element", lambda self, call, name, t: kgq.F32, raising=False)
    monkeypatch.setattr(kgq.Engine, "_matrix", lambda self, call, name, t, width=None: (kgq.F32, t.stride(0)))
    monkeypatch.setattr(kgq.Engine, "_array", lambda *a: None)
    e = kgq.Engine(kgq.GQE, 50, 6, 8, 12.0, 4, device=-1)
    e.device = 0                                               # (what streams are asked for; the handle has none)
    return e


class CallersStream:
    cuda_stream = 4096


class Copies(torch.utils._python_dispatch.TorchDispatchMode):
    """The copies that are made, each with the stream that it is made on."""

    def __init__(self, on):
        super().__init__()
        self.on, self.made = on, []

    def __torch_dispatch__(self, func, types, args=(), kwargs=None):
        if func.overloadpacket.__name__ in COPIES:
            self.made.append(self.on[-1])
        return func(*args, **(kwargs or {}))


BEYOND = (1 << 32) + 5                                         # 5, if cut to 32 bits


@pytest.mark.parametrize("what", ["embed ids", "embed columns", "embed_grad ids", "embed_grad columns", "sample rows",
                                  "sample draws", "sample top_k", "distill rows", "distill k"])
def test_sizes_beyond_32_bits_are_refused(eng, monkeypatch, what):
    """Counts that the library takes as 32-bit integers are not cut to them."""
    monkeypatch.setattr(torch, "empty", lambda *a, **k: pytest.fail("memory asked for"))
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: None)
    f = lambda *shape: torch.zeros(1).expand(*shape)
    i = lambda *shape: torch.zeros(1, dtype=torch.int32).expand(*shape)
    call = {
        "embed ids": lambda s: eng.embed(f(4, 8), i(BEYOND), stream=s),
        "embed columns": lambda s: eng.embed(f(1, BEYOND), i(3), stream=s),
        "embed_grad ids": lambda s: eng.embed_grad(f(BEYOND, 8), i(BEYOND), 10, stream=s),
        "embed_grad columns": lambda s: eng.embed_grad(f(3, BEYOND), i(3), 10, stream=s),
        "sample rows": lambda s: eng.sample(f(BEYOND, 50), f(BEYOND, 3), stream=s),
        "sample draws": lambda s: eng.sample(f(2, 50), f(2, BEYOND), stream=s),
        "sample top_k": lambda s: eng.sample(f(2, 50), f(2, 3), top_k=BEYOND, stream=s),
        "distill rows": lambda s: eng.distill(f(BEYOND, 50), i(BEYOND, 3), f(BEYOND, 3), stream=s),
        "distill k": lambda s: eng.distill(f(2, 50), i(2, BEYOND), f(2, BEYOND), stream=s),
    }[what]
    with pytest.raises(ValueError, match="32 bits"):
        call(CallersStream())


@pytest.mark.parametrize("layout", ["rows cut off", "transposed", "flat"])
def test_a_gradients_copy_is_made_on_the_calls_stream(eng, monkeypatch, layout):
    """A gradient whose rows have no common stride is copied; the kernels run
    behind that copy only if both are on one stream."""
    on = [None]

    @contextlib.contextmanager
    def stream(s):
        on.append(s)
        yield
        on.pop()

    kept = []
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: kept.append((t, s)))
    grad = {"rows cut off": torch.zeros(4, 6, 8)[:, 1:], "transposed": torch.zeros(5, 4, 8).transpose(0, 1),
            "flat": torch.zeros(4, 5, 8)}[layout]
    ids = torch.zeros(4, 5, dtype=torch.int32)
    mine = CallersStream()
    with Copies(on) as copies, pytest.raises(kgq.KgqError) as e:
        eng.embed_grad(grad, ids, 10, stream=mine)
    assert e.value.name == "NO_DEVICE"                         # everything else passed
    assert copies.made == ([] if layout == "flat" else [mine])
    # the caller's own memory outlives the work on it
    assert any(t.data_ptr() == grad.data_ptr() and s is mine for t, s in kept)


def distill_into(eng, monkeypatch, scores, out):
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: None)
    monkeypatch.setattr(torch.cuda, "stream", lambda s: contextlib.nullcontext())
    B = scores.shape[0]
    idx, score = torch.zeros(B, 3, dtype=torch.int32), torch.zeros(B, 3)
    eng.distill(scores, idx, score, out=out, stream=CallersStream())


def test_distill_out_may_share_a_buffer_with_scores(eng, monkeypatch):
    """Column ranges that share no element are not refused, ranges that share
    one are; so are rows that interleave with another stride."""
    buf = torch.zeros(4, 130)
    flat = torch.zeros(4 * 130 + 200)
    rows = lambda at, ld: torch.as_strided(flat, (4, 50), (ld, 1), at)
    apart = [(buf[:, :50], buf[:, 50:100]), (buf[:, 80:], buf[:, 30:80]), (buf[:, :50], buf[:, 80:]),
             (rows(0, 130), rows(180, 130)),                   # a column range, a row on
             (rows(0, 130), rows(80, 130)),                    # up to the next row's start
             (rows(0, 50), rows(200, 50)), (buf[:, :50], buf[:, :50]), (buf[:1, :50], buf[1:2, 20:70])]
    met = [(buf[:, :50], buf[:, 49:99]), (buf[:, 49:99], buf[:, :50]), (rows(0, 130), rows(129, 130)),
           (rows(0, 130), rows(81, 130)), (rows(0, 130), rows(130, 130)), (rows(0, 50), rows(150, 50)),
           (rows(0, 100), rows(50, 101)), (rows(0, 100), rows(0, 101)), (buf[:1, :50], buf[:1, 49:99])]
    for expected, pairs in (("NO_DEVICE", apart), ("overlaps", met)):
        for scores, out in pairs:
            cells = [{int(i) for i in torch.as_strided(torch.arange(10 ** 4), t.shape, t.stride(), t.storage_offset()).flatten()}
                     for t in (scores, out)]
            same = cells[0] == cells[1] and scores.stride() == out.stride()
            if scores.stride() == out.stride() or scores.shape[0] == 1:
                assert (same or not cells[0] & cells[1]) == (expected == "NO_DEVICE")     # (the lists above are right)
            with pytest.raises((kgq.KgqError, ValueError), match=expected):
                distill_into(eng, monkeypatch, scores, out)
