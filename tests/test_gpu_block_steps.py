"""append_decode on a block-scaled cache: outputs and bytes of append and decode, whether or
not a block fills; its refusals change nothing.
"""
import numpy as np
import pytest

from paper_2607_16248_amd import BlockCache, KvqError, kvq

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

B, HKV, GQ, CAP = 3, 2, 4, 700
HQ = HKV * GQ


def images(c):
    return [c.export(s, h) for s in range(B) for h in range(HKV)]


def pair(**kw):
    return [BlockCache(B, HQ, HKV, CAP, **kw) for _ in range(2)]


@pytest.mark.parametrize("kw", [dict(type_k="e4m3", block_tokens=32), dict(type_k="i8", type_v="e4m3", block_tokens=64, fp16_window=40),
                                dict(type_k="i8", block_tokens=32, fp16_window=7, page_tokens=128)])
def test_steps(kw):
    a, b = pair(**kw)
    g = torch.Generator(device="cuda").manual_seed(1)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda").half()  # noqa: E731
    K, V = rnd(B, 400, HKV, 128), rnd(B, 400, HKV, 128)
    for c in (a, b):
        c.append(K, V, [400, 63, 0])
    held, side = [400, 63, 0], torch.cuda.Stream()
    for step in range(70):  # (every sequence fills a block on the way)
        n = 1 if step % 10 else 5
        new = [n, 1, n] if step % 7 else [n, 0, 1]
        k, v, q = rnd(B, n, HKV, 128), rnd(B, n, HKV, 128), rnd(B, HQ, 128)
        if step % 5 == 4:  # (a workspace of the call's own, on another stream)
            side.wait_stream(torch.cuda.current_stream())
            got = a.append_decode(k, v, q, new, stream=side)
            torch.cuda.current_stream().wait_stream(side)
        else:
            got = a.append_decode(k, v, q, new)
        b.append(k, v, new)
        assert torch.equal(got, b.decode(q)), step
        held = [x + y for x, y in zip(held, new)]
        assert [a.seq_len(s) for s in range(B)] == held
    assert all(np.array_equal(x, y) for x, y in zip(images(a), images(b)))
    a.check()


def test_a_step_without_tokens_is_a_decode():
    a, b = pair(type_k="i8")
    x = torch.randn((B, 90, HKV, 128), device="cuda").half()
    q = torch.randn((B, HQ, 128), device="cuda").half()
    for c in (a, b):
        c.append(x, x, [90, 0, 31])
    got = a.append_decode(x[:, :1].contiguous(), x[:, :1].contiguous(), q, [0, 0, 0])
    assert torch.equal(got, b.decode(q)) and not got[1].any()
    assert all(np.array_equal(x, y) for x, y in zip(images(a), images(b)))


def test_refusals_change_nothing():
    """Counts, capacity, pages and a workspace that is too small: lengths and bytes stay, and the step works afterwards."""
    a, b = (BlockCache(B, HQ, HKV, CAP, "i8", page_tokens=128, num_pages=8) for _ in range(2))
    x = torch.randn((B, 600, HKV, 128), device="cuda").half()
    q, out = torch.randn((B, HQ, 128), device="cuda").half(), torch.zeros((B, HQ, 128), device="cuda")
    for c in (a, b):
        c.append(x, x, [600, 255, 0])  # (pages: 5 of 576 packed tokens, 2 of 192: one is left)
    ws = torch.empty(kvq.kvq_workspace_bytes(a.handle), dtype=torch.uint8, device="cuda")
    before = images(a)
    for n, n_max, size, status in (((2, 0, 0), 1, None, kvq.ERR_ARG), ((101, 0, 0), 200, None, kvq.ERR_CAPACITY),
                                   ((0, 129, 200), 200, None, kvq.ERR_CAPACITY), ((1, 1, 1), 1, 16, kvq.ERR_CAPACITY)):
        with pytest.raises(KvqError) as e:
            kvq.kvq_append_decode(a.handle, x, x, n, q, out, ws, size, n_max=n_max)
        assert e.value.status == status
        assert [a.seq_len(s) for s in range(B)] == [600, 255, 0]
        assert all(np.array_equal(u, v) for u, v in zip(before, images(a)))
    k = x[:, :1].contiguous()
    kvq.kvq_append_decode(a.handle, k, k, (1, 1, 1), q, out, ws)
    b.append(k, k, [1, 1, 1])
    assert torch.equal(out, b.decode(q))


def test_the_smallest_workspace():
    """The smallest size that a decode takes is enough and kept to; one byte less is refused."""
    c = BlockCache(2, HQ, HKV, 3000, "i8", block_tokens=32, fp16_window=16)
    x = torch.randn((2, 3000, HKV, 128), device="cuda").half()
    c.append(x, x, [3000, 20])
    q = torch.randn((2, HQ, 128), device="cuda").half()
    want = c.decode(q)
    top = kvq.kvq_workspace_bytes(c.handle)
    buf = torch.full((top + 64,), 0x5A, dtype=torch.uint8, device="cuda")
    out = torch.empty_like(want)

    def taken(size):
        try:
            kvq.kvq_decode_attention(c.handle, q, out, buf, size)
            return True
        except KvqError as e:
            assert e.status == kvq.ERR_CAPACITY
            return False

    low, high = 0, top  # (refused, taken)
    assert taken(top) and not taken(0)
    while high - low > 1:
        mid = (low + high) // 2
        low, high = (low, mid) if taken(mid) else (mid, high)
    torch.cuda.synchronize()
    buf.fill_(0x5A)
    out.fill_(float("nan"))
    assert taken(high) and not taken(high - 1)
    torch.cuda.synchronize()
    assert torch.equal(out, want) and (buf[high:] == 0x5A).all()
