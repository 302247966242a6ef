"""Block-scaled caches beyond 4 GiB: a head that begins there, pages that lie there, attention
over all of it against 64 bits.

Bound of an output: that of test_gpu_block.py, and the roundings of long sums: a wave adds a
weight sum and an accumulator once per 32 tokens; with 170 workgroups of four waves per head
at least that is n / 32 / 680 + 8 additions one after another, each off by 2^-24 of the sum
(of |V^| by weight for the numerator), and 16 more where waves and parts are joined.
"""
import math

import pytest

from paper_2607_16248_amd import BlockCache

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

HKV, GQ, N, PART = 3, 2, 9_000_000, 500_000


@pytest.mark.parametrize("page", [0, 4096])
def test_heads_and_pages_past_4_gib(page):
    if torch.cuda.mem_get_info()[0] < 20 << 30:
        pytest.skip("not enough device memory")
    c = BlockCache(1, GQ * HKV, HKV, N, "i8", "e4m3", block_tokens=128, page_tokens=page)
    # contiguous: the last head's keys, scales and values all begin past 2^32
    assert page or c.arena.numel() // HKV * (HKV - 1) > 1 << 32
    assert c.arena.numel() > 6 << 30
    g = torch.Generator(device="cuda").manual_seed(1)
    q = torch.randn((1, GQ * HKV, 128), generator=g, device="cuda").half()
    far = N - 700_000  # a block whose keys answer the first query of every kv head, far behind in each of them
    for k in range(0, N, PART):
        x, v = (torch.randn((1, min(PART, N - k), HKV, 128), generator=g, device="cuda").half() for _ in range(2))
        if k <= far < k + PART:
            for h in range(HKV):
                x[0, far - k:far - k + 64, h] += 2 * q[0, GQ * h]
        c.append(x, v)
    c.check()
    out = c.decode(q).double()
    # the values read back, in parts: running maximum, sums of weights, of values and of their magnitudes
    top = torch.full((GQ * HKV,), -math.inf, device="cuda", dtype=torch.float64)
    mass, num, size = (torch.zeros((GQ * HKV,) + s, device="cuda", dtype=torch.float64) for s in ((), (128,), (128,)))
    most = torch.zeros((), device="cuda", dtype=torch.float64)
    for k in range(0, N, PART):
        K, V = (x.double() for x in c.dequant(0, k, min(PART, N - k)))
        for h in range(GQ * HKV):
            kh, vh, qh = K[:, h // GQ].contiguous(), V[:, h // GQ].contiguous(), q[0, h].double()
            s = kh @ qh * (math.log2(math.e) / math.sqrt(128))
            most = torch.maximum(most, (kh.abs() @ qh.abs()).max() * (math.log2(math.e) / math.sqrt(128)))
            m = torch.maximum(top[h], s.max())
            w, f = torch.exp2(s - m), torch.exp2(top[h] - m)
            top[h], mass[h] = m, mass[h] * f + w.sum()
            num[h], size[h] = num[h] * f + w @ vh, size[h] * f + w @ vh.abs()
        del K, V
    ref, size = num / mass[:, None], size / mass[:, None]
    chain = 2 * (N / 32 / 680 + 8 + 16) * 2.0 ** -24
    tol = 2 * math.log(2) * 16 * 2.0 ** -24 * float(most) + 2.0 ** -20 + chain
    # (weights off by 2^-33 of the largest: at most 2^-31 n |V^|, |V^| below 8, by the largest weight, 1 / mass)
    bound = tol * size + 2.0 ** -31 * N * 8 / mass[:, None]
    err = (out[0] - ref).abs()
    assert bool((err <= bound).all()), float((err / bound).max())
    # the block that answers is what the first queries see, 64 values' mean by weight
    first = ref[::GQ]
    assert float(first.abs().max()) > 0.05 and float(bound[::GQ].max()) < 0.2 * float(first.abs().max())
