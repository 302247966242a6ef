"""Block-scaled caches whose blocks or fp16 tail hold values of zero alone: what the other
tokens give keeps its bits, however far the zeros' scores lie above theirs.

Bounds are those of test_gpu_block.py (Setup.check).  A block of zeros stands in a row's
reference as one of scale 2^-80, so weights are off by up to 2^-33 2^-80 of its own: with
leads up to 2^70 that is 2^-43 of the others' sum at most, inside the 2^-20 that are
allowed.
"""
import numpy as np
import pytest

from paper_2607_16248_amd import kvq
from test_gpu_block import Setup

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def run(s, q, name):
    n_q = q.shape[1]
    qd = torch.from_numpy(q).cuda()
    if n_q == 1:
        s.check(q, s.cache.decode(qd), name=(name, "decode"))
    s.check(q, s.cache.chunk(qd), name=(name, "chunk"))
    for window, sinks in ((70, 0), (1 << 30, 0), (50, 33)):
        s.check(q, s.cache.window(qd, window, sinks), window, sinks, name=(name, window, sinks))


@pytest.mark.parametrize("n_q", [1, 6, 8, 40, 70])
@pytest.mark.parametrize("kinds", [("e4m3", "i8"), ("i8", "e4m3")])
@pytest.mark.parametrize("power", [0, -12, -15])
def test_a_block_of_the_tail_without_values(n_q, kinds, power):
    """Zeros in a block of the tail (a head that wrote nothing there), values of 2^power before and behind it, ordinary
    scores."""
    rng = np.random.default_rng(n_q)
    n, R = 32 * 6 + 20, 100  # (96 packed tokens, 116 in the tail)
    K, V = 0.5 * rng.standard_normal((1, n, 2, 128)), 2.0 ** power * rng.standard_normal((1, n, 2, 128))
    for first in (96, 128):
        V[:, first:first + 32] = 0.0
        s = Setup([n], *kinds, gq=4, R=R, kv=(K.astype(np.float16), V.astype(np.float16)))
        run(s, s.queries(n_q, 0.25), first)


@pytest.mark.parametrize("n_q", [1, 6, 8, 40])
@pytest.mark.parametrize("kind", ["e4m3", "i8"])
@pytest.mark.parametrize("lead", [1.0, 2.0, 3.0, 4.2])
@pytest.mark.parametrize("at", [0, 3])
def test_a_block_of_zeros_far_above(n_q, kind, lead, at):
    """A packed block of zero values whose scores lead by about 16 lead (base 2): 16 to 67."""
    rng = np.random.default_rng(7)
    n = 32 * 18 + 9  # (every wave of a tile has several blocks)
    u = rng.choice([-1.0, 1.0], (128,))
    K, V = 0.1 * rng.standard_normal((1, n, 2, 128)), rng.standard_normal((1, n, 2, 128))
    K[:, 32 * at:32 * at + 32] = u * lead / 2
    V[:, 32 * at:32 * at + 32] = 0.0
    s = Setup([n], kind, gq=4, kv=(K.astype(np.float16), V.astype(np.float16)))
    kvq.kvq_set_split_tokens(s.cache.handle, 32 * 20)  # (one part)
    q = (2.0 * u + 0.1 * rng.standard_normal((1, n_q, s.hq, 128))).astype(np.float16)
    run(s, q, (lead, at))


def test_many_blocks_of_zeros():
    """Sums of weights that stand for 2^80 each stay in range: 25000 tokens of zeros, and one block with values."""
    n = 32 * 800
    rng = np.random.default_rng(3)
    K, V = rng.standard_normal((1, n, 1, 128)).astype(np.float16), np.zeros((1, n, 1, 128), np.float16)
    V[:, 32 * 300:32 * 301] = rng.standard_normal((1, 32, 1, 128))
    s = Setup([n], "e4m3", gq=4, hkv=1, kv=(K, V))
    for n_q in (1, 5, 40):
        q = s.queries(n_q)
        for split in (0, 32 * 400):
            kvq.kvq_set_split_tokens(s.cache.handle, split)
            s.cache.ws = None
            s.check(q, s.cache.chunk(torch.from_numpy(q).cuda()), name=(n_q, split))
