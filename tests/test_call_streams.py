"""The tensors that a call of KVCache makes for itself belong to the stream that its
kernels run on (no GPU needed: torch's allocator and streams are stood in for).

A freed tensor's memory goes to the next tensor of the stream that it was made on.  A
workspace made on the current stream for kernels of another one, and dropped when the
call returns, is the current stream's next tensor's while those kernels still use it.
"""
import contextlib

import pytest

from paper_2607_16248_amd import kvq

torch = pytest.importorskip("torch")


class Stream:
    def __init__(self, name, handle):
        self.name, self.cuda_stream = name, handle

    def __repr__(self):
        return self.name


CURRENT, OTHER, DEFAULT = Stream("current", 16), Stream("other", 32), Stream("default", 0)


class Log:
    def __init__(self):
        self.scope = [CURRENT]
        self.made = []      # (stream, shape)
        self.recorded = []  # (shape, stream)
        self.calls = []     # stream argument of the library's call


@pytest.fixture
def log(monkeypatch):
    x = Log()
    empty = torch.empty

    @contextlib.contextmanager
    def stream(s):
        x.scope.append(s)
        try:
            yield
        finally:
            x.scope.pop()

    def make(shape, **kw):
        t = empty(shape, **kw)
        x.made.append((x.scope[-1], tuple(t.shape)))
        return t

    monkeypatch.setattr(torch.cuda, "is_available", lambda: True)
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: x.scope[-1])
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device=None: DEFAULT)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device=None: {32: OTHER, 16: CURRENT}[handle])
    monkeypatch.setattr(torch, "empty", make)
    monkeypatch.setattr(torch.Tensor, "is_cuda", True)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: x.recorded.append((tuple(t.shape), s)))
    for name in ("kvq_window_workspace_bytes", "kvq_chunk_workspace_bytes", "kvq_workspace_bytes"):
        monkeypatch.setattr(kvq, name, lambda *a: 5000)
    for name in ("kvq_window_attention", "kvq_chunk_attention", "kvq_decode_attention", "kvq_append_decode"):
        monkeypatch.setattr(kvq, name, lambda *a, stream=None, **kw: x.calls.append(stream))
    return x


def cache():
    c = object.__new__(kvq.KVCache)
    c.batch, c.num_q_heads, c.head_dim, c.handle, c.ws, c.ws_stream = 2, 8, 128, None, None, None
    c.arena = torch.zeros(1, dtype=torch.uint8)
    return c


Q = torch.zeros((2, 3, 8, 128), dtype=torch.half)
OUT = (2, 3, 8, 128)


@pytest.mark.parametrize("given,runs_on", [(OTHER, OTHER), (32, OTHER), (0, DEFAULT), (CURRENT, CURRENT), (None, CURRENT)], ids=str)
def test_window_makes_its_tensors_on_the_stream_it_runs_on(log, given, runs_on):
    cache().window(Q, 8, 2, stream=given)
    assert sorted(log.made, key=str) == sorted([(runs_on, OUT), (runs_on, (5000,))], key=str)
    assert log.calls == [given] and log.scope == [CURRENT]
    if runs_on is not CURRENT:  # the output is the caller's, who is on the current stream
        assert log.recorded == [(OUT, CURRENT)]
    # an output of the caller's stays as it is
    log.made.clear()
    log.recorded.clear()
    cache().window(Q, 8, 2, out=torch.zeros(OUT), stream=given)
    assert log.made == [(runs_on, (5000,))] and log.recorded == []


CALLS = {"chunk": (OUT, lambda c, **kw: c.chunk(Q, **kw)), "decode": (OUT[:1] + OUT[2:], lambda c, **kw: c.decode(Q[:, 0], **kw)),
         "append_decode": (OUT[:1] + OUT[2:], lambda c, **kw: c.append_decode(Q, Q, Q[:, 0], **kw))}


@pytest.mark.parametrize("call", list(CALLS))
@pytest.mark.parametrize("given,runs_on", [(OTHER, OTHER), (32, OTHER), (0, DEFAULT), (None, CURRENT)], ids=str)
def test_the_other_calls_do_too(log, call, given, runs_on):
    shape, f = CALLS[call]
    c = cache()
    f(c, stream=given)
    assert sorted(log.made, key=str) == sorted([(runs_on, shape), (runs_on, (5000,))], key=str)
    assert log.recorded == ([(shape, CURRENT)] if given is not None else [])
    handle = {None: 16, OTHER: 32}.get(given, given)
    assert log.calls in ([given], [handle])


@pytest.mark.parametrize("call", ["decode", "append_decode"])
def test_the_caches_workspace_stays_with_its_stream(log, call):
    shape, f = CALLS[call]
    c = cache()
    f(c)
    assert log.made.count((CURRENT, (5000,))) == 1
    for given in (None, CURRENT):  # kept
        log.made.clear()
        f(c, stream=given)
        assert log.made == [(CURRENT, shape)]
    log.made.clear()
    f(c, stream=OTHER)
    assert (OTHER, (5000,)) in log.made
    with torch.cuda.stream(OTHER):  # the current stream is another one now
        log.made.clear()
        f(c)
        assert (OTHER, (5000,)) in log.made
        log.made.clear()  # the workspace's stream by name, not the current one: nothing of the current one's
        f(c, stream=CURRENT)
        assert {s for s, _ in log.made} == {CURRENT}
    log.made.clear()
    f(c)
    assert log.made == [(CURRENT, shape)]
