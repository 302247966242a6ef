"""GPU parity of kvq_window_attention (a sliding window and the first tokens)
against the fp64 oracle on the same quantized cache, through the public calls.

Every output has to lie within
    tol * softmax-weighted M of its channel,  tol = 2 ln 2 * 16 * 2^-24 * A + 2^-20,
M a token's largest |V^| in the channel's value group: V^ = z + code s is the
sum of (z + c0 s) and (code - c0) s, neither of them larger than 2 M, each held
to 22 bits or more, so that a value that comes out near zero is as exact as its
group's largest and no more (2^-24 M for each of the two, and for their sums).
A is the largest sum_c |q_c K^_c| log2(e) / sqrt(d) of the row's tokens: a score
is a sum of 128 fp32-accumulated products (16 roundings at its magnitude
allowed), an error d of base-2 scores moves a weight and the sum of weights by
ln 2 * d each, and weights, keys and values enter with 22 bits or more
(2^-20 for all of them).  That is about 4e-5 for these inputs.
"""
import math

import numpy as np
import pytest

import oracle
from paper_2607_16248_amd import KvqError, kvq
from workloads import Workload, gen_kv

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

HQ_HKV = {1: (2, 2), 2: (4, 2), 4: (8, 2), 5: (10, 2), 8: (8, 1)}


class Setup:
    """A cache of ragged sequences, its inputs, and the oracle's dequantized heads."""

    def __init__(self, lens, bk, bv, gq=4, gk=32, gv=32, R=0, page=0, cap=0, seed=11, kmul=1.0, vmul=1.0, vadd=0.0):
        self.hq, self.hkv = HQ_HKV[gq]
        b = len(lens)
        bk, bv = ([x] * b if isinstance(x, int) else list(x) for x in (bk, bv))
        self.lens, self.bk, self.bv, self.gk, self.gv, self.R = lens, bk, bv, gk, gv, R
        cap = cap or max(max(lens), 1)
        self.cache = kvq.KVCache(b, self.hq, self.hkv, cap, bk, bv, key_group=gk, value_group=gv, fp16_window=R,
                                 page_tokens=page)
        w = Workload("window", b, self.hq, self.hkv, 128, tuple(lens), tuple(bk), tuple(bv), gk, gv, R, cfg_id=seed)
        self.kv = [gen_kv(w, 0, s) for s in range(b)]
        if (kmul, vmul, vadd) != (1.0, 1.0, 0.0):
            self.kv = [((k * np.float32(kmul)).astype(np.float16), (v * np.float32(vmul) + np.float32(vadd)).astype(np.float16))
                       for k, v in self.kv]
        n = max(max(lens), 1)
        K, V = (np.zeros((b, n, self.hkv, 128), dtype=np.float16) for _ in range(2))
        for s, (k, v) in enumerate(self.kv):
            K[s, :lens[s]], V[s, :lens[s]] = k, v
        if max(lens) > 0:
            self.cache.append(torch.from_numpy(K).cuda(), torch.from_numpy(V).cuda(), list(lens))
        self.rng = np.random.default_rng([seed, b, max(lens)])

    def queries(self, n_q):
        return self.rng.standard_normal((len(self.lens), n_q, self.hq, 128)).astype(np.float16)

    def dequant(self, s):
        K, V = self.kv[s]
        out = []
        for h in range(self.hkv):
            args = (self.bk[s], self.bv[s], self.gk, self.gv, self.R)
            img = oracle.build_head(np.ascontiguousarray(K[:, h]), np.ascontiguousarray(V[:, h]), *args)
            out.append(oracle.dequant_head(img, self.lens[s], 128, *args))
        return np.stack([x[0] for x in out]), np.stack([x[1] for x in out])

    def check(self, q, got, window, sinks, only=None):
        worst = 0.0
        assert np.isfinite(got).all()
        for s, n in enumerate(self.lens):
            if only is not None and s not in only:
                continue
            if n == 0:
                assert (got[s] == 0).all()
                continue
            Kh, Vh = self.dequant(s)
            ref = oracle.window_attention(q[s], Kh, Vh, window, sinks)
            M = np.abs(Vh).reshape(self.hkv, n, 128 // self.gv, self.gv).max(-1).repeat(self.gv, -1)
            size = oracle.window_attention(q[s], Kh, M, window, sinks)
            k = np.abs(Kh).repeat(self.hq // self.hkv, 0)
            A = (np.abs(q[s].astype(np.float64)).transpose(1, 0, 2) @ k.transpose(0, 2, 1)).max() * math.log2(math.e) / math.sqrt(128)
            tol = 2 * math.log(2) * 16 * 2.0 ** -24 * A + 2.0 ** -20
            err = np.abs(got[s] - ref) / size
            worst = max(worst, err.max() / tol)
            assert (err <= tol).all(), (s, n, np.unravel_index(err.argmax(), err.shape), err.max(), tol)
        return worst


def run(c, q, window, sinks):
    out = torch.full(q.shape, float("nan"), dtype=torch.float32, device="cuda")
    got = c.cache.window(torch.from_numpy(q).cuda(), window, sinks, out=out)
    torch.cuda.synchronize()
    return got.cpu().numpy()


CASES = [
    # single tokens: ragged batches with an empty slot, a single token, windows of 1, inside the tail, past the length
    ("one_token", dict(lens=(1,), bk=2, bv=2), 1, 1, 0),
    ("ragged_empty", dict(lens=(0, 1, 31, 33, 700), bk=2, bv=2), 1, 100, 4),
    ("window_1", dict(lens=(500, 64), bk=1, bv=1), 1, 1, 0),
    ("window_1_sink_1", dict(lens=(500, 64), bk=4, bv=4), 1, 1, 1),
    ("window_past_length", dict(lens=(333, 90), bk=2, bv=1), 1, 1 << 30, 0),
    ("all_sinks", dict(lens=(333, 90), bk=8, bv=8), 1, 5, 1 << 30),
    ("window_in_tail", dict(lens=(700, 130), bk=2, bv=2, R=128), 1, 20, 0),
    ("window_in_tail_sinks", dict(lens=(700, 130), bk=2, bv=2, R=128), 1, 20, 37),
    ("sinks_in_tail", dict(lens=(100, 60), bk=2, bv=2, R=100), 1, 10, 25),
    ("sinks_across_packed_end", dict(lens=(160, 165), bk=2, bv=2, R=100), 1, 10, 70),
    ("only_tail_long", dict(lens=(400,), bk=1, bv=1, R=400), 1, 65, 3),
    ("gq5_gk64", dict(lens=(900, 257), bk=8, bv=8, gq=5, gk=64, R=17), 1, 311, 16),
    ("gq8_gk128", dict(lens=(1000, 640), bk=4, bv=8, gq=8, gk=128, gv=64), 1, 300, 5),
    ("gq1_fine", dict(lens=(700, 300), bk=2, bv=2, gq=1, gv=16, R=5), 1, 222, 1),
    ("gq2_mixed_class", dict(lens=(700, 300), bk=1, bv=4, gq=2, gv=8), 1, 222, 40),
    ("mixed_batch", dict(lens=(600, 64, 999, 5), bk=(1, 2, 4, 8), bv=(8, 1, 4, 2), R=40), 1, 150, 4),
    ("paged", dict(lens=(900, 10, 513), bk=4, bv=4, page=64, R=32), 1, 200, 70),
    ("paged_gk128", dict(lens=(900, 10, 513), bk=2, bv=2, gk=128, gv=128, page=128), 1, 130, 4),
    # several queries: each with a window of its own
    ("verify5", dict(lens=(700, 33), bk=4, bv=2, R=128), 5, 64, 4),
    ("verify3_gq5", dict(lens=(700, 301), bk=2, bv=2, gq=5), 3, 33, 0),
    ("whole_sequence", dict(lens=(48,), bk=1, bv=1), 48, 7, 2),
    ("chunk_64", dict(lens=(1100,), bk=2, bv=2, R=32), 64, 100, 4),
    ("chunk_64_short_window", dict(lens=(600,), bk=8, bv=8, gk=128), 64, 3, 0),
    ("chunk_200_gq1", dict(lens=(500,), bk=1, bv=1, gq=1), 200, 40, 37),
    ("chunk_130_gq8", dict(lens=(700, 131), bk=4, bv=4, gq=8, gk=64), 130, 150, 1),
    ("chunk_150_paged", dict(lens=(700, 400), bk=2, bv=2, page=64, R=64), 150, 90, 33),
    ("chunk_90_mixed", dict(lens=(500, 140, 700), bk=(1, 8, 4), bv=(4, 8, 4), R=10), 90, 128, 4),
]


@pytest.mark.parametrize("name,kw,n_q,window,sinks", CASES, ids=[c[0] for c in CASES])
def test_window_matches_oracle(name, kw, n_q, window, sinks):
    print(f"[window] {name}", flush=True)
    c = Setup(**kw)
    q = c.queries(n_q)
    got = run(c, q, window, sinks)
    c.cache.check()
    worst = c.check(q, got, window, sinks)
    print(f"[window] {name}: largest error / tolerance {worst:.3f}", flush=True)
    again = run(c, q, window, sinks)
    assert (got.view(np.uint32) == again.view(np.uint32)).all()


@pytest.mark.parametrize("bk,bv", [(1, 1), (1, 2), (2, 1), (2, 2), (4, 4), (4, 8), (8, 4), (8, 8), (1, 4), (8, 2), (2, 8), (4, 1), (1, 8),
                                   (8, 1), (4, 2), (2, 4)])
def test_every_class(bk, bv):
    c = Setup((420, 77), bk, bv, R=3)
    q = c.queries(1)
    c.check(q, run(c, q, 100, 4), 100, 4)
    for n_q in (30, 70):  # 16-row groups, many rows
        q = c.queries(n_q)
        c.check(q, run(c, q, 50, 4), 50, 4)


@pytest.mark.parametrize("kw", [dict(vmul=1e-5), dict(vmul=2e-7), dict(vadd=3000.0), dict(vmul=5000.0), dict(kmul=1e-5),
                                dict(kmul=20.0), dict(vmul=1e-3, vadd=1e-4)], ids=str)
@pytest.mark.parametrize("bits", [1, 2, 4, 8])
def test_small_and_large_numbers(kw, bits):
    # scales and zero-points that are subnormal halves, values far from zero, keys that peak the softmax
    c = Setup((330, 200), bits, bits, R=20, **kw)
    for n_q in (1, 6, 70):
        q = c.queries(n_q)
        c.check(q, run(c, q, 120, 4), 120, 4)


@pytest.mark.parametrize("kw", [dict(vmul=2e-7), dict(vmul=5000.0), dict(kmul=1e-5), dict(vadd=3000.0)], ids=str)
@pytest.mark.parametrize("bk,bv", [(1, 4), (2, 8), (4, 2), (8, 1)])
def test_small_and_large_numbers_of_mixed_bits(kw, bk, bv):
    # keys of one or two fp16 parts beside values of the other
    c = Setup((330, 200), bk, bv, R=20, **kw)
    q = c.queries(70)
    c.check(q, run(c, q, 120, 4), 120, 4)


def check_many(lens, n_q, window, sinks, **kw):
    """Windows of a batch that keeps every compute unit busy, where long chunks take 256 rows per workgroup: the
    sequences `lens` and short ones beside them."""
    more = tuple(n_q + 20 + i % 60 for i in range(64 - len(lens)))
    both = {x: kw.pop(x) for x in ("bk", "bv")}
    c = Setup(tuple(lens) + more, both["bk"], both["bv"], **kw)
    q = c.queries(n_q)
    c.check(q, run(c, q, window, sinks), window, sinks, only=(*range(len(lens)), 40, 63))


@pytest.mark.parametrize("bk", [1, 2, 4, 8])
@pytest.mark.parametrize("bv", [1, 2, 4, 8])
def test_many_rows_every_class(bk, bv):
    check_many((420, 77), 70, 50, 4, bk=bk, bv=bv, R=3)


@pytest.mark.parametrize("kw", [dict(vmul=1e-5), dict(vmul=2e-7), dict(vadd=3000.0), dict(vmul=5000.0), dict(kmul=1e-5),
                                dict(kmul=20.0), dict(vmul=1e-3, vadd=1e-4)], ids=str)
@pytest.mark.parametrize("bk,bv", [(1, 1), (8, 8), (2, 4), (4, 2)])
def test_many_rows_small_and_large_numbers(kw, bk, bv):
    check_many((330, 200), 70, 120, 4, bk=bk, bv=bv, R=20, **kw)


@pytest.mark.parametrize("n_q,window,sinks,lens,kw", [
    (70, 100, 4, (900, 71, 513), dict(bk=4, bv=4, page=64, R=32)),
    (70, 130, 4, (900, 70), dict(bk=2, bv=2, gk=128, gv=128, page=128)),
    (200, 40, 37, (500, 200), dict(bk=1, bv=1, gq=1)),
    (100, 90, 0, (500, 333), dict(bk=2, bv=8, gq=2, gv=64)),
    (70, 33, 3, (700, 301), dict(bk=2, bv=2, gq=5)),
    (70, 150, 1, (700, 131), dict(bk=4, bv=4, gq=8, gk=64)),
    (70, 1, 0, (300, 96), dict(bk=2, bv=2)),
    (70, 1, 1, (300, 96), dict(bk=8, bv=4, R=17)),
    (70, 20, 90, (250, 140), dict(bk=2, bv=2, R=100)),
    (70, 1 << 30, 0, (400, 70), dict(bk=2, bv=1, R=64)),
    (70, 64, 1 << 30, (400, 90), dict(bk=1, bv=4)),
    (70, 30, 4, (260, 75), dict(bk=2, bv=2, R=300))], ids=lambda x: str(x).replace(" ", ""))
def test_many_rows_layouts_and_masks(n_q, window, sinks, lens, kw):
    check_many(lens, n_q, window, sinks, **kw)


@pytest.mark.parametrize("n,n_q", [(64, 1), (65, 1), (130, 1), (67, 4)])
def test_more_sequences_than_a_launch_describes(n, n_q):
    lens = [n_q + (37 * i) % 150 for i in range(n)]
    c = Setup(tuple(lens), [(1, 2, 4, 8)[i % 4 if n == 130 else 1] for i in range(n)], 2, gq=1, R=33)
    q = c.queries(n_q)
    c.check(q, run(c, q, 60, 4), 60, 4)


def test_few_queries_over_long_and_short_sequences():
    # one sequence of many splits beside one of a single split, in and out of the tail's own workgroups
    for lens, window in (((9000, 12), 8192), ((9000, 12, 40, 3000), 4096), ((20000,), 20000)):
        c = Setup(lens, 2, 4, R=64)
        q = c.queries(1)
        c.check(q, run(c, q, window, 4), window, 4)


def test_forced_splits_and_growing_cache():
    # every length around a key group's end, splits of one and of two groups
    c = Setup((60,), 2, 2, R=8, cap=200)
    w = Workload("grow", 1, c.hq, c.hkv, 128, (140,), (2,), (2,), 32, 32, 8, cfg_id=12)
    K, V = gen_kv(w, 0, 0)
    K[:60], V[:60] = c.kv[0]
    for n in range(60, 138, 3):
        c.cache.append(torch.from_numpy(K[None, n:n + 3]).cuda(), torch.from_numpy(V[None, n:n + 3]).cuda())
        c.kv, c.lens = [(K[:n + 3], V[:n + 3])], (n + 3,)
        kvq.kvq_set_split_tokens(c.cache.handle, 32 * (1 + n % 2))
        q = c.queries(2)
        c.check(q, run(c, q, 40, 5), 40, 5)


def test_captured_and_replayed_on_another_stream():
    c = Setup((700, 300), 2, 2, R=16)
    window, sinks = 100, 4
    q = c.queries(1)
    qd = torch.from_numpy(q).cuda()
    out = torch.zeros((2, 1, c.hq, 128), device="cuda")
    want = run(c, q, window, sinks)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        c.cache.window(qd, window, sinks, out=out)
    s.synchronize()
    assert (out.cpu().numpy().view(np.uint32) == want.view(np.uint32)).all()
    # two graphs of the same cache, replayed in turn with eager work between
    graphs = []
    for nq in (1, 3):
        x = torch.from_numpy(c.queries(nq)).cuda()
        y = torch.zeros((2, nq, c.hq, 128), device="cuda")
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c.cache.window(x, window, sinks, out=y)
        graphs.append((g, x, y))
    for _ in range(3):
        for g, x, y in graphs:
            fresh = c.queries(x.shape[1])
            x.copy_(torch.from_numpy(fresh))
            y.fill_(float("nan"))
            g.replay()
            torch.cuda.synchronize()
            eager = run(c, fresh, window, sinks)
            assert (y.cpu().numpy().view(np.uint32) == eager.view(np.uint32)).all()


def test_two_streams_at_once():
    a, b = Setup((900, 400), 2, 2, seed=13), Setup((500, 777), 4, 4, R=20, seed=14)
    qs = [a.queries(1), b.queries(40)]
    want = [run(a, qs[0], 200, 4), run(b, qs[1], 64, 2)]
    dev = [torch.from_numpy(q).cuda() for q in qs]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(5):
        outs = []
        for c, q, st, (w, k) in zip((a, b), dev, streams, ((200, 4), (64, 2))):
            with torch.cuda.stream(st):
                outs.append(c.cache.window(q, w, k))
        torch.cuda.synchronize()
        for o, x in zip(outs, want):
            assert (o.cpu().numpy().view(np.uint32) == x.view(np.uint32)).all()


def test_wide_window_agrees_with_full_attention():
    c = Setup((700, 133), 8, 2, R=30)
    q = c.queries(20)
    full = c.cache.chunk(torch.from_numpy(q).cuda()).cpu().numpy()
    c.check(q, full, 1 << 20, 0)
    c.check(q, run(c, q, 1 << 20, 0), 1 << 20, 0)


def test_guard_bands():
    guard, pattern = 1 << 16, 0xA5
    c = Setup((900, 333), 2, 2, R=24)
    for n_q, window, sinks in ((1, 64, 4), (7, 300, 0), (100, 64, 40)):
        q = c.queries(n_q)
        bufs = []
        for n in (q.size * 4, kvq.kvq_window_workspace_bytes(c.cache.handle, n_q, window, sinks)):
            bufs.append(torch.full((n + 2 * guard,), pattern, dtype=torch.uint8, device="cuda"))
        out, ws = (b[guard:b.numel() - guard] for b in bufs)
        kvq.kvq_window_attention(c.cache.handle, torch.from_numpy(q).cuda(), n_q, window, sinks, out, ws)
        torch.cuda.synchronize()
        for b in bufs:
            assert bool((b[:guard] == pattern).all()) and bool((b[-guard:] == pattern).all())
        c.check(q, out.view(torch.float32).view(q.shape).cpu().numpy(), window, sinks)


def test_refusals_leave_the_output():
    c = Setup((10, 40), 2, 2)
    q = torch.zeros((2, 1, c.hq, 128), dtype=torch.half, device="cuda")
    out = torch.full((2, 1, c.hq, 128), 7.0, device="cuda")
    ws = torch.empty(kvq.kvq_window_workspace_bytes(c.cache.handle, 1, 8, 0), dtype=torch.uint8, device="cuda")
    for n_q, window, sinks, w in ((0, 8, 0, ws), (1, 0, 0, ws), (1, 8, -1, ws), (11, 8, 0, ws), (1, 8, 0, ws[:16]),
                                  (1, 8, 0, ws[4:]), (1, 8, 0, None), (1025, 8, 0, ws)):
        with pytest.raises(KvqError):
            kvq.kvq_window_attention(c.cache.handle, q, n_q, window, sinks, out, w)
    torch.cuda.synchronize()
    assert bool((out == 7.0).all())
