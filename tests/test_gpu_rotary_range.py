"""Rotated appends of numbers that do not fit fp16: reported where they enter the cache, the
fp16 window too, before anything is packed.  (Queries are the caller's and are not looked at.)
"""
import numpy as np
import pytest

from paper_2607_16248_amd import BlockCache, KVCache, KvqError, kvq
from test_gpu_rotary import tables

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

N, WINDOW = 40, 64  # (all tokens stay in the window)
CACHES = {"k4v4": lambda **kw: KVCache(2, 4, 2, 300, [4] * 2, [4] * 2, key_group=32, fp16_window=WINDOW, **kw),
          "k1v8": lambda **kw: KVCache(2, 4, 2, 300, [1] * 2, [8] * 2, key_group=64, fp16_window=WINDOW, **kw),
          "e4m3": lambda **kw: BlockCache(2, 4, 2, 300, "e4m3", block_tokens=32, fp16_window=WINDOW, **kw),
          "i8": lambda **kw: BlockCache(2, 4, 2, 300, "i8", block_tokens=128, fp16_window=WINDOW, **kw)}


def reported(c):
    try:
        c.check()
        return False
    except KvqError as e:
        assert e.status == kvq.ERR_RANGE
        return True


def rows(dtype):
    g = torch.Generator(device="cuda").manual_seed(2)
    return [torch.randn((2, N, h, 128), generator=g, device="cuda").to(dtype) for h in (4, 2, 2)]


@pytest.mark.parametrize("kind", list(CACHES))
@pytest.mark.parametrize("page", [0, 128])
@pytest.mark.parametrize("rot,pairs", [(128, False), (64, True)])
def test_tokens_of_the_window(kind, page, rot, pairs):
    cos, sin = (torch.from_numpy(t).cuda() for t in tables(300, rot))
    for dtype, value in ((torch.bfloat16, 70000.0), (torch.bfloat16, -3e38), (torch.float16, float("inf")),
                         (torch.bfloat16, float("nan"))):
        for which, at in ((None, None), (1, (0, 0, 0, 0)), (1, (1, N - 1, 1, 127)), (2, (0, 17, 1, 64)), (2, (1, 33, 0, 3)),
                          (0, (0, 5, 3, 9))):
            x = rows(dtype)
            if which is not None:
                x[which][at] = value
            c = CACHES[kind](page_tokens=page)
            c.append_rotary(*x, cos, sin, pairs=pairs)
            assert reported(c) == (which in (1, 2)), (dtype, value, which, at)
            c.reset()
            assert not reported(c)


@pytest.mark.parametrize("kind", list(CACHES))
def test_a_turn_past_the_range(kind):
    """Finite halves whose rotated pair is larger than any half; the same pair a quarter turn on fits."""
    for angle, out in ((np.pi / 4, True), (np.pi / 2, False)):
        cos, sin = (torch.full((300, 64), f(angle), device="cuda") for f in (np.cos, np.sin))
        q, k, v = rows(torch.float16)
        k[1, 30, 0, 7], k[1, 30, 0, 71] = 60000.0, 60000.0
        c = CACHES[kind]()
        c.append_rotary(q, k, v, cos, sin)
        assert reported(c) == out


@pytest.mark.parametrize("kind", list(CACHES))
def test_rows_behind_the_new_tokens_are_not_read(kind):
    cos, sin = (torch.from_numpy(t).cuda() for t in tables(300, 128))
    q, k, v = rows(torch.bfloat16)
    k[0, 3:], v[1, 20:] = float("inf"), float("nan")
    c = CACHES[kind]()
    c.append_rotary(q, k, v, cos, sin, [3, 20])
    assert not reported(c)
    c.append_rotary(*(x[:, 2:4].contiguous() for x in (q, k, v)), cos, sin, [2, 0])  # (token 3 of the first one: infinite)
    assert reported(c)
