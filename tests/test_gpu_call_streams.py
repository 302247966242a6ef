"""KVCache's calls with their ``stream`` argument: a stream other than the current one,
with allocations and other calls on the current stream between them.  Results are those
of the same calls on the current stream, bit by bit.
"""
import numpy as np
import pytest

from paper_2607_16248_amd import kvq

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_window import Setup  # noqa: E402


def bits(x):
    return x.cpu().numpy().view(np.uint32)


def others(c):
    """Streams a call may name, none of them the current one."""
    s = [torch.cuda.Stream(), torch.cuda.Stream()]
    return s + [s[0].cuda_stream, s[1].cuda_stream]


CALLS = {"window": lambda c, q, **kw: c.window(q, 200, 4, **kw), "chunk": lambda c, q, **kw: c.chunk(q, **kw),
         "decode": lambda c, q, **kw: c.decode(q, **kw)}


@pytest.mark.parametrize("call", list(CALLS))
def test_on_a_named_stream(call):
    print(f"[streams] {call}", flush=True)
    c = Setup((3000, 700), 2, 2, R=40, seed=21)
    n_q = (1, 5, 70) if call in ("window", "chunk") else (1,)
    qs = [torch.from_numpy(c.queries(n)).cuda() for n in n_q]
    if call not in ("window", "chunk"):
        qs = [q[:, 0].contiguous() for q in qs]
    f = CALLS[call]
    want = [bits(f(c.cache, q)) for q in qs]
    torch.cuda.synchronize()
    streams = others(c)
    for turn in range(3):
        got = []
        for n, s in enumerate(streams):
            for q in qs:
                out = f(c.cache, q, stream=s)
                # what the current stream makes and writes meanwhile is not the calls' memory
                held = [torch.full((x,), float("nan"), device="cuda") for x in (1 << 10, 1 << 14, 1 << 18, 1 << 20)]
                f(c.cache, q)
                got.append((n, out, held))
        torch.cuda.synchronize()
        for i, (n, out, _) in enumerate(got):
            assert (bits(out) == want[i % len(qs)]).all(), (turn, n, i)


def test_workspace_is_not_the_next_tensors(monkeypatch):
    c = Setup((3000, 700), 2, 2, R=40, seed=22)
    q = torch.from_numpy(c.queries(5)).cuda()
    seen = []
    real = kvq.kvq_window_attention

    def call(*a, **kw):
        seen.append((a[6].data_ptr(), a[6].numel()))
        return real(*a, **kw)

    monkeypatch.setattr(kvq, "kvq_window_attention", call)
    c.cache.window(q, 200, 4)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        c.cache.window(q, 200, 4, stream=s)
        at, size = seen[-1]
        x = torch.empty((size,), dtype=torch.uint8, device="cuda")
        assert x.data_ptr() >= at + size or x.data_ptr() + size <= at
    torch.cuda.synchronize()


def test_decode_steps_on_two_streams_at_once():
    # one cache, two streams: each step has a workspace of its own
    c = Setup((60000, 30000), 2, 2, R=40, seed=23)
    qs = [torch.from_numpy(c.queries(1)[:, 0].copy()).cuda() for _ in range(2)]
    want = [bits(c.cache.decode(q)) for q in qs]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(10):
        outs = []
        for q, s in zip(qs, streams):
            with torch.cuda.stream(s):
                outs.append(c.cache.decode(q))
        outs += [c.cache.decode(qs[0], stream=streams[1]), c.cache.decode(qs[1])]
        torch.cuda.synchronize()
        for out, w in zip(outs, want + want):
            assert (bits(out) == w).all()
