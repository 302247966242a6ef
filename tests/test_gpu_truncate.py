"""kvq_truncate on packed caches: every call after it, against a cache that never held the
dropped tokens (bit for bit) and against attention over the values that the cache reads
back, in 64 bits.

Tolerances: windows, whose weights enter the products in two halves, are within 1e-5
(2-norm) by their header.  Decode and chunk weights of the matrix kernels enter as one
half: each is off by up to 2^-11 of itself, so an output by up to 2^-11 sum_t w_t |V^_t -
out|; over tokens of random signs, where sum_t w_t |V^_t| is up to four times the row's
largest output at these lengths, that is 2e-3 of it, the bound that these calls have
everywhere (ATTN_TOL, row-normwise).
"""
import math

import numpy as np
import pytest

from helpers import ATTN_TOL
from paper_2607_16248_amd import KVCache, KvqError, kvq

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

HKV = 2
CLASSES = [  # bits, key group, value group, fp16 window, page, heads per kv head
    ((1, 1), 32, 32, 40, 0, 4), ((2, 2), 64, 32, 64, 128, 5), ((4, 4), 32, 32, 33, 256, 4), ((8, 8), 128, 64, 96, 0, 8),
    ((2, 8), 32, 32, 50, 0, 2), ((4, 8), 64, 16, 70, 128, 1)]


def make(bits, gk, gv, R, page, gq, cap=1500, batch=2):
    return KVCache(batch, gq * HKV, HKV, cap, [bits[0]] * batch, [bits[1]] * batch, key_group=gk, value_group=gv, fp16_window=R,
                   page_tokens=page)


def images(c):
    return [c.export(s, h) for s in range(c.batch) for h in range(HKV)]


def same(a, b):
    return all(np.array_equal(x, y) for x, y in zip(images(a), images(b)))


def check(c, q, out, window=None, sinks=0):
    """Attention over the values read back."""
    n_q, gq = q.shape[1], c.num_q_heads // HKV
    out = out.reshape(c.batch, n_q, c.num_q_heads, 128).double().cpu()
    for s in range(c.batch):
        L = c.seq_len(s)
        K, V = (x.double().cpu() for x in c.dequant(s, 0, L))
        pos, t = torch.arange(L - n_q, L)[:, None], torch.arange(L)
        vis = t <= pos
        if window is not None:
            vis = vis & ((t > pos - window) | (t < sinks))
        for h in range(c.num_q_heads):
            x = q[s, :, h].double().cpu() @ K[:, h // gq].t().contiguous() / math.sqrt(128)
            ref = torch.softmax(x.masked_fill(~vis, -math.inf), 1) @ V[:, h // gq].contiguous()
            err = out[s, :, h] - ref
            worst = float((err.norm(dim=1) / ref.norm(dim=1)).max()) if window else \
                float((err.abs().amax(1) / ref.abs().amax(1)).max())
            assert worst <= (1e-5 if window else ATTN_TOL), (s, h, n_q, window, worst)


class Run:
    def __init__(self, cls, lens, seed=1):
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        self.a, self.b = make(*cls), make(*cls)
        self.gq = cls[5]
        n = max(lens)
        x = self.rows(n), self.rows(n)
        for c in (self.a, self.b):
            c.append(*x, lens)

    def rows(self, n, heads=HKV):
        return torch.randn((2, n, heads, 128), generator=self.g, device="cuda").half()

    def attend(self, twin):
        """Every attention call of the cache that was cut back, against 64 bits (and bit for bit against its twin)."""
        for n_q in (1, 3, 9, 40, 130):
            if n_q > min(self.a.seq_len(s) for s in range(2)):
                break
            q = self.rows(n_q, self.gq * HKV)
            calls = [lambda c: c.chunk(q), lambda c: c.window(q, 60, 5), lambda c: c.window(q, 300)]
            if n_q == 1:
                calls.append(lambda c: c.decode(q[:, 0].contiguous()))
            outs = [f(self.a) for f in calls]
            for out, (w, k) in zip(outs, ((None, 0), (60, 5), (300, 0), (None, 0))):
                check(self.a, q, out, w, k)
            if twin:
                assert all(torch.equal(o, f(self.b)) for o, f in zip(outs, calls))


@pytest.mark.parametrize("cls", CLASSES)
def test_drafts_that_fill_no_group(cls):
    """What is left has the bytes and results of a cache that never grew, and grows on like it."""
    gk, R = cls[1], cls[3]
    lens = [R + 3 * gk + 2, R + 5 * gk + 1]
    r = Run(cls, lens)
    for n in (1, 7, gk - 4):
        junk = r.rows(n)
        r.a.append(junk, junk)
        r.a.truncate(lens)
        assert [r.a.seq_len(s) for s in range(2)] == lens and same(r.a, r.b)
    r.attend(True)
    for n in (1, 1, 2, gk, 2 * gk + 5):
        k, v, q = r.rows(n), r.rows(n), r.rows(1, r.gq * HKV)[:, 0].contiguous()
        assert torch.equal(r.a.append_decode(k, v, q), r.b.append_decode(k, v, q))
    assert same(r.a, r.b)
    r.a.check()


@pytest.mark.parametrize("cls", CLASSES)
def test_packed_groups_stay(cls):
    """Drafts that fill groups: cut back to the packed tokens at most, fewer than the window behind them.  Attention is
    over what the cache holds; tokens appended again give the bytes of a cache that was never cut back."""
    gk, R = cls[1], cls[3]
    lens = [R + 2 * gk, R + 4 * gk + 3]
    r = Run(cls, lens)
    k, v = r.rows(2 * gk + 5), r.rows(2 * gk + 5)
    for c in (r.a, r.b):
        c.append(k, v)
    packed = [(n + 2 * gk + 5 - R) // gk * gk for n in lens]
    for cut in ([packed[0], packed[1] + 1], [packed[0], packed[1]]):
        r.a.truncate(cut)
        assert [r.a.seq_len(s) for s in range(2)] == cut
        with pytest.raises(KvqError) as e:
            r.a.truncate([cut[0], packed[1] - 1])
        assert e.value.status == kvq.ERR_STATE
        r.attend(False)
    # the dropped tokens once more, some by decode steps, some by appends
    full = torch.zeros((2, 4 * gk + R, HKV, 128), device="cuda", dtype=torch.float16)
    left = [n + 2 * gk + 5 - p for n, p in zip(lens, packed)]
    K, V = full.clone(), full.clone()
    for s in range(2):
        # (what the window still held of the first append is read back from the twin)
        x, y = r.b.dequant(s, packed[s], left[s])
        K[s, :left[s]], V[s, :left[s]] = x.half(), y.half()
    done = [0, 0]
    for n in (1, 1, 3, R + gk):
        new = [min(n, m - d) for m, d in zip(left, done)]
        kn, vn = full[:, :n].clone(), full[:, :n].clone()
        for s in range(2):
            kn[s, :new[s]], vn[s, :new[s]] = K[s, done[s]:done[s] + new[s]], V[s, done[s]:done[s] + new[s]]
        q = r.rows(1, r.gq * HKV)
        out = r.a.append_decode(kn, vn, q[:, 0].contiguous(), new)
        check(r.a, q, out)
        done = [d + m for d, m in zip(done, new)]
    assert done == left and same(r.a, r.b)
    k, v = r.rows(gk + 9), r.rows(gk + 9)
    for c in (r.a, r.b):
        c.append(k, v)
    assert same(r.a, r.b)
    r.attend(True)
    r.a.check()


def test_released_and_cut_back():
    """A sequence cut back to nothing before anything was packed; a released one takes another's place."""
    r = Run(CLASSES[2], [20, 20])
    r.a.truncate([0, 20])
    assert not r.a.decode(r.rows(1, 4 * HKV)[:, 0].contiguous())[0].any()
    k, v = r.rows(100), r.rows(100)
    r.a.append(k, v, [100, 0])
    r.b.release(0)
    r.b.append(k, v, [100, 0])
    assert same(r.a, r.b)
    r.a.release(1)
    r.b.release(1)
    for c in (r.a, r.b):
        c.append(k, v, [0, 70])
    assert same(r.a, r.b)
    r.attend(True)
