"""Block-scaled attention where scales lie far apart: weights keep their bits beside blocks
whose largest values the row's tokens have no part in.

Bound of an output: that of test_gpu_block.py with each part as it is here,
    (2 ln 2 * 16 * 2^-24 A + 2^-17) sum_t w_t |V^_t| + 2^-31 n max_t w_t m_t.
log2 of a scale (magnitudes below 64) is off by 2^-18 at most, its sum with a reference and
an exponent by half of that each, which moves a weight by ln 2 * 2^-17, and 22-bit weights
and sums stay below the rest of 2^-17.  n: the row's visible tokens; m_t: the largest
magnitude of token t's block of one scale, visible or not (of the fp16 tail: of 32 tokens).
A weight times its scale is off by 2^-33 of the row's largest such product, and a value is at
most 448 of its scale (tail: 256 of a power of two), a scale 1/127 of its block's largest:
448 / 127 * 2^-33 < 2^-31.
"""
import math

import numpy as np
import pytest

from block_oracle import attention, packed_len
from test_gpu_block import Setup

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def check(s, q, out, window=None, sinks=0, name=""):
    out, n_q = out.cpu().numpy(), q.shape[1]
    out = out.reshape(len(s.lens), n_q, s.hq, 128)
    for i, L in enumerate(s.lens):
        pos, t, p = np.arange(L - n_q, L)[:, None], np.arange(L), packed_len(L, s.block, s.R)
        vis = t <= pos
        if window is not None:
            vis &= (t > pos - window) | (t < sinks)
        for h in range(s.hkv):
            k, v = s.held(i, h)
            top = np.abs(v).max(1)
            m = np.concatenate([top[:p].reshape(-1, s.block).max(1).repeat(s.block),
                                np.pad(top[p:], (0, -(L - p) % 32)).reshape(-1, 32).max(1).repeat(32)[:L - p]])
            for g in range(s.gq):
                x = q[i, :, h * s.gq + g]
                ref, mass, size = attention(x, k, v, vis)
                w, _, _ = attention(x, k, np.eye(L), vis)
                tol = 2 * math.log(2) * 16 * 2.0 ** -24 * size + 2.0 ** -17
                bound = tol[:, None] * mass + (2.0 ** -31 * vis.sum(1) * (w * m).max(1))[:, None]
                err = np.abs(out[i, :, h * s.gq + g] - ref)
                assert (err <= bound).all(), (name, i, h, g, float((err / np.maximum(bound, 1e-300)).max()))


@pytest.mark.parametrize("n_q,gq", [(1, 8), (6, 4), (12, 8), (40, 4), (60, 8)])
@pytest.mark.parametrize("power", [-14, -8, -3, 4])
@pytest.mark.parametrize("kind", ["i8", "e4m3"])
def test_a_tail_beside_a_large_scale(n_q, gq, power, kind):
    """Zeros behind values of 1000 in the last packed block, a tail of values of 2^power: the windows see the zeros and the tail."""
    rng = np.random.default_rng(n_q)
    n = 128 + 60
    K, V = 0.3 * rng.standard_normal((1, n, 1, 128)), rng.standard_normal((1, n, 1, 128))
    V[:, 64:96], V[:, 96:128], V[:, 128:] = 1000.0 * V[:, 64:96], 0.0, 2.0 ** power * V[:, 128:]
    s = Setup([n], kind, gq=gq, hkv=1, block=64, R=32, kv=(K.astype(np.float16), V.astype(np.float16)))
    assert packed_len(n, 64, 32) == 128
    for scale in (0.0, 0.3, 2.0):
        q = s.queries(n_q, scale)
        qd = torch.from_numpy(q).cuda()
        for window in (n - 96, 90, 64, 1 << 30):
            check(s, q, s.cache.window(qd, window), window, 0, name=(scale, window))
        check(s, q, s.cache.chunk(qd), name=scale)


@pytest.mark.parametrize("seed", range(24))
def test_scales_of_all_sizes(seed):
    """Runs of 32 tokens between 2^-16 and 2^10, of zeros, of keys without size; ragged, paged, split; windows and sinks."""
    from paper_2607_16248_amd import kvq
    rng = np.random.default_rng(seed)
    b, block, R = int(rng.choice([1, 2, 3])), int(rng.choice([32, 64, 128])), int(rng.choice([0, 5, 32, 70, 200]))
    gq, hkv, n_q = int(rng.choice([1, 2, 4, 5, 8])), int(rng.choice([1, 2])), [1, 3, 8, 13, 24, 33, 60, 140][seed % 8]
    lens = [int(n) for n in rng.integers(n_q, n_q + 400, b)]
    L = max(lens)
    K, V = rng.standard_normal((b, L, hkv, 128)), rng.standard_normal((b, L, hkv, 128))
    for i in range(b):
        for h in range(hkv):
            for t in range(0, L, 32):
                V[i, t:t + 32, h] *= [1.0, 0.0, 2.0 ** rng.integers(-16, 11), 1.0][rng.integers(0, 4)]
                K[i, t:t + 32, h] *= [1.0, 1.0, 2.0 ** rng.integers(-8, 1), 0.0][rng.integers(0, 4)]
    s = Setup(lens, str(rng.choice(["i8", "e4m3"])), str(rng.choice(["i8", "e4m3"])), gq=gq, hkv=hkv, block=block, R=R,
              page=int(rng.choice([0, 128])), kv=(K.astype(np.float16), V.astype(np.float16)))
    q = s.queries(n_q, float(rng.choice([0.05, 0.5, 1.0])))
    qd = torch.from_numpy(q).cuda()
    for split in (0, block, 3 * block):
        kvq.kvq_set_split_tokens(s.cache.handle, split)
        check(s, q, s.cache.chunk(qd), name=split)
        for window, sinks in ((1, 4), (30, 0), (30, 40), (100, 130)):
            check(s, q, s.cache.window(qd, window, sinks), window, sinks, name=(split, window, sinks))
