"""Block-scaled caches on the GPU: bytes against the 64-bit quantizer, attention
(decode, chunk, window) against 64-bit attention over the same values, through the
public calls.

Every output has to lie within
    tol * sum_t w_t |V^_t|,  tol = 2 ln 2 * 16 * 2^-24 * A + 2^-20
of its channel: A is the largest sum_c |q_c K^_c| log2(e) / sqrt(d) of the row's tokens
(a score is a sum of 128 products accumulated in fp32, 16 roundings at its magnitude
allowed; an error d of base-2 scores moves a weight and the sum of weights by ln 2 * d
each); weights enter with 22 bits, keys and values exactly, and a scale's way through
the exponent costs 2^-22 (2^-20 for all of them).  A weight's low half is a multiple of
2^-24 where the row's largest weight times its block's scale is 2^8 at least, so each
weight times scale is off by up to 2^-25 / 2^8 of that largest one, however small it is
itself: a token's value is at most 448 of its scale, a scale at most 1/127 of its block's
largest value m, and n tokens add
    n * 448 / 127 * 2^-33 * max_t w_t m_t  <  2^-31 n max_t w_t m_t
(what is left where every token of weight has the value 0 in a channel).
"""
import math

import numpy as np
import pytest

from block_oracle import attention, cached, head_image, packed_len, quantize_blocks, zero_signs
from paper_2607_16248_amd import BlockCache, KvqError, kvq

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


class Setup:
    """A block-scaled cache of ragged sequences and what it was given."""

    def __init__(self, lens, tk="e4m3", tv=None, gq=4, hkv=2, block=32, R=0, page=0, cap=0, seed=3, chunks=None, kv=None,
                 num_pages=0):
        self.lens, self.tk, self.tv, self.block, self.R = list(lens), tk, tv or tk, block, R
        self.hq, self.hkv, self.gq = gq * hkv, hkv, gq
        b, n = len(lens), max(max(lens), 1)
        self.rng = np.random.default_rng([seed, b, n])
        if kv is None:
            K = self.rng.standard_normal((b, n, hkv, 128)) * np.where(self.rng.random((b, 1, hkv, 128)) < 0.03, 10.0, 1.0)
            kv = K.astype(np.float16), self.rng.standard_normal((b, n, hkv, 128)).astype(np.float16)
        self.K, self.V = kv
        self.cache = BlockCache(b, self.hq, hkv, cap or n, tk, self.tv, block_tokens=block, fp16_window=R, page_tokens=page,
                                num_pages=num_pages)
        at = [0] * b
        for step in chunks or [n]:
            new = [min(step, L - p) for L, p in zip(lens, at)]
            if max(new) == 0:
                continue
            m = max(new)
            k, v = (np.zeros((b, m, hkv, 128), np.float16) for _ in range(2))
            for i in range(b):
                k[i, :new[i]], v[i, :new[i]] = self.K[i, at[i]:at[i] + new[i]], self.V[i, at[i]:at[i] + new[i]]
            self.cache.append(torch.from_numpy(k).cuda(), torch.from_numpy(v).cuda(), new)
            at = [p + n for p, n in zip(at, new)]
        assert at == self.lens
        torch.cuda.synchronize()

    def queries(self, n_q, scale=1.0):
        return (scale * self.rng.standard_normal((len(self.lens), n_q, self.hq, 128))).astype(np.float16)

    def held(self, s, h):
        L = self.lens[s]
        return cached(self.K[s, :L, h], self.V[s, :L, h], self.tk, self.tv, self.block, self.R)

    def check(self, q, out, window=None, sinks=0, name=""):
        out = out.cpu().numpy() if not isinstance(out, np.ndarray) else out
        n_q = q.shape[1]
        out = out.reshape(len(self.lens), n_q, self.hq, 128)
        for s, L in enumerate(self.lens):
            if L == 0:
                assert not out[s].any()
                continue
            pos = np.arange(L - n_q, L)[:, None]
            t = np.arange(L)
            vis = t <= pos
            if window is not None:
                vis &= (t > pos - window) | (t < sinks)
            for h in range(self.hkv):
                k, v = self.held(s, h)
                for g in range(self.gq):
                    ref, mass, size = attention(q[s, :, h * self.gq + g], k, v, vis)
                    tol = 2 * math.log(2) * 16 * 2.0 ** -24 * size + 2.0 ** -20
                    most = np.abs(np.pad(v, ((0, -L % 32), (0, 0)))).reshape(-1, 32 * 128).max(1).repeat(32)[:L]
                    _, reach, _ = attention(q[s, :, h * self.gq + g], k, np.diag(most) if L <= 512 else most[:, None], vis)
                    reach = reach.max(1) if L <= 512 else reach[:, 0]  # (the sum is more than the largest)
                    bound = tol[:, None] * mass + 2.0 ** -31 * L * reach[:, None]
                    err = np.abs(out[s, :, h * self.gq + g] - ref)
                    assert (err <= bound).all(), (name, s, h, g, float((err / bound).max()))


def images(c, lens, hkv):
    return [[c.export(s, h) for h in range(hkv)] for s in range(len(lens))]


@pytest.mark.parametrize("tk,tv", [("i8", "i8"), ("e4m3", "e4m3"), ("i8", "e4m3")])
@pytest.mark.parametrize("block,R,page", [(32, 0, 0), (64, 40, 0), (128, 5, 256), (32, 130, 128)])
def test_bytes_and_values(tk, tv, block, R, page):
    lens = [1, 31, 200, 333, 0]
    for chunks in (None, [7, 100, 1, 1, 150, 400], [1] * 34 + [400]):
        s = Setup(lens, tk, tv, block=block, R=R, page=page, chunks=chunks)
        for i, L in enumerate(lens):
            for h in range(s.hkv):
                want = head_image(s.K[i, :L, h], s.V[i, :L, h], tk, tv, block, R)
                got = s.cache.export(i, h)
                assert got.shape == want.shape
                assert np.array_equal(zero_signs(got, tk, tv, block, R, L), zero_signs(want, tk, tv, block, R, L))
            if L == 0:
                continue
            for t0, n in ((0, L), (L // 3, L - L // 3), (L - 1, 1)):
                Kd, Vd = (x.cpu().numpy() for x in s.cache.dequant(i, t0, n))
                for h in range(s.hkv):
                    k, v = s.held(i, h)
                    assert np.array_equal(Kd[:, h], k[t0:t0 + n].astype(np.float32))
                    assert np.array_equal(Vd[:, h], v[t0:t0 + n].astype(np.float32))
        s.cache.check()


def special_blocks(kind):
    """Blocks of 32 tokens where codes are easily wrong: ties, borders of the type's steps, tiny and huge numbers."""
    top = {"i8": 127.0, "e4m3": 448.0}[kind]
    rng = np.random.default_rng(1)
    blocks = []
    for s in (1.0, 2.0 ** -7, 2.0 ** -12, 64.0 if kind == "e4m3" else 256.0):  # scale s exactly: every tie is a number of fp16's
        if kind == "i8":
            x = (rng.integers(-254, 255, (32, 128)) / 2.0) * s
        else:
            grid = np.array([m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10) for e in range(16) for m in range(8)][:127])
            mids = np.concatenate([grid, (grid[1:] + grid[:-1]) / 2])
            x = rng.choice(mids, (32, 128)) * rng.choice([-1.0, 1.0], (32, 128)) * s
        x[0, 0] = top * s
        blocks.append(x)
    blocks.append(np.zeros((32, 128)))                                  # nothing
    blocks.append(np.full((32, 128), 2.0 ** -24))                       # the smallest number
    blocks.append(rng.integers(-3, 4, (32, 128)) * 2.0 ** -24)          # subnormal ones
    blocks.append(rng.uniform(-65504, 65504, (32, 128)))                # the largest
    one = np.zeros((32, 128))
    one[7, 77] = -65504.0                                               # one large among none
    blocks.append(one)
    blocks.append(np.where(rng.random((32, 128)) < 0.01, 1000.0, 1e-3 * rng.standard_normal((32, 128))))
    for top_x in (3.0, 0.7, 1234.0):                                    # every fp16 number up to the largest, near all borders
        x = rng.integers(0, int(np.float16(top_x).view(np.uint16)) + 1, (32, 128)).astype(np.uint16).view(np.float16).astype(np.float64)
        x[3, 3] = top_x
        blocks.append(x * rng.choice([-1.0, 1.0], (32, 128)))
    return np.stack(blocks).astype(np.float16)


@pytest.mark.parametrize("kind", ["i8", "e4m3"])
def test_codes_at_ties_and_extremes(kind):
    x = special_blocks(kind).reshape(1, -1, 1, 128)
    n = x.shape[1]
    s = Setup([n], kind, gq=1, hkv=1, kv=(x, x[:, ::-1].copy()))
    got, want = s.cache.export(0, 0), head_image(x[0, :, 0], x[0, ::-1, 0], kind, kind, 32, 0)
    assert np.array_equal(zero_signs(got, kind, kind, 32, 0, n), zero_signs(want, kind, kind, 32, 0, n))
    s.cache.check()


@pytest.mark.parametrize("value", [np.inf, -np.inf, np.nan])
def test_elements_that_are_not_finite(value):
    K, V = np.ones((1, 96, 2, 128), np.float16), np.ones((1, 96, 2, 128), np.float16)
    K[0, 40, 1, 5] = value
    s = Setup([96], "i8", gq=1, kv=(K, V))
    with pytest.raises(KvqError) as e:
        s.cache.check()
    assert e.value.status == kvq.ERR_RANGE
    Kd, Vd = (x.cpu().numpy() for x in s.cache.dequant(0, 0, 96))
    assert not Kd[32:64, 1].any() and (Vd == 1).all() and (Kd[:, 0] == 1).all() and (Kd[64:, 1] == 1).all()
    s.cache.reset()
    s.cache.check()


CASES = [  # lens, kinds, heads per kv head, block, window, page
    ([1], "i8", "i8", 4, 32, 0, 0), ([33, 5, 0, 64], "e4m3", "i8", 5, 32, 0, 0), ([700, 31], "i8", "e4m3", 8, 64, 37, 128),
    ([1500, 1, 129, 640], "e4m3", "e4m3", 2, 128, 130, 256), ([2100], "i8", "i8", 1, 32, 64, 0),
    ([5000, 40, 2222], "e4m3", "e4m3", 4, 64, 0, 0), ([300] * 9, "i8", "e4m3", 5, 64, 128, 128),
]


@pytest.mark.parametrize("lens,tk,tv,gq,block,R,page", CASES)
def test_decode(lens, tk, tv, gq, block, R, page):
    s = Setup(lens, tk, tv, gq=gq, block=block, R=R, page=page)
    q = s.queries(1)
    out = s.cache.decode(torch.from_numpy(q).cuda())
    s.check(q, out)
    no_ws = torch.empty_like(out)
    kvq.kvq_decode_attention_noalloc(s.cache.handle, torch.from_numpy(q).cuda(), no_ws)
    assert torch.equal(no_ws.view(-1), out.view(-1))
    for split in (block, 3 * block, 2048):
        kvq.kvq_set_split_tokens(s.cache.handle, split)
        s.cache.ws = None
        s.check(q, s.cache.decode(torch.from_numpy(q).cuda()), name=split)


@pytest.mark.parametrize("n_q", [2, 3, 5, 7, 13, 16, 17, 33, 65, 130])
@pytest.mark.parametrize("tk,tv,gq,block,R,page", [("i8", "e4m3", 4, 32, 0, 128), ("e4m3", "e4m3", 5, 64, 70, 0),
                                                   ("i8", "i8", 8, 128, 200, 0), ("e4m3", "i8", 1, 32, 32, 0)])
def test_chunks_and_windows(n_q, tk, tv, gq, block, R, page):
    lens = [n_q, n_q + 1, n_q + 300, n_q + 77]
    s = Setup(lens, tk, tv, gq=gq, block=block, R=R, page=page)
    q = s.queries(n_q)
    qd = torch.from_numpy(q).cuda()
    s.check(q, s.cache.chunk(qd), name="chunk")
    for window, sinks in ((1, 0), (33, 4), (100, 40), (1 << 30, 0), (5, 1 << 30)):
        s.check(q, s.cache.window(qd, window, sinks), window, sinks, name=(window, sinks))
    kvq.kvq_set_split_tokens(s.cache.handle, block)
    s.check(q, s.cache.chunk(qd), name="split")


@pytest.mark.parametrize("n_q", [1, 6, 40])
def test_scales_far_apart(n_q):
    """Neighbouring blocks whose values (and keys) differ by up to 2^20, blocks of zeros, numbers of the fp16 tail below
    2^-14 and above 8: each row's small values keep their bits where the large ones have no weight."""
    rng = np.random.default_rng(5)
    n = 32 * 12 + 20
    K, V = rng.standard_normal((1, n, 1, 128)), rng.standard_normal((1, n, 1, 128))
    for b in range(13):
        V[0, 32 * b:32 * b + 32] *= [1.0, 2.0 ** -10, 0.0, 512.0, 2.0 ** -12, 3.0, 2.0 ** 10, 2.0 ** -3, 0.0, 8.0, 2.0 ** -6, 1.0, 2.0 ** -15][b]
        K[0, 32 * b:32 * b + 32] *= [1.0, 0.0, 2.0 ** -8, 4.0, 1.0, 2.0 ** -14, 0.5, 1.0, 1.0, 0.0, 8.0, 1.0, 1.0][b]
    V[0, n - 3] *= 2.0 ** 20
    s = Setup([n], "e4m3", "i8", gq=4, hkv=1, kv=(K.astype(np.float16), V.astype(np.float16)))
    for scale in (1.0, 2.0 ** -20, 30.0):
        q = s.queries(n_q, scale)
        s.check(q, s.cache.chunk(torch.from_numpy(q).cuda()), name=scale)
        s.check(q, s.cache.window(torch.from_numpy(q).cuda(), 2), 2, 0, name=("window", scale))


def test_queries_of_zero():
    s = Setup([200, 40], "i8", R=16)
    for n_q in (1, 3, 33):
        q = np.zeros((2, n_q, s.hq, 128), np.float16)
        s.check(q, s.cache.chunk(torch.from_numpy(q).cuda()))


def test_truncate_and_grow_again():
    """Rejected drafts: a cache that grew, was cut back and grew on holds the bytes of one that never did."""
    for block, R in ((32, 40), (64, 64)):
        a = Setup([300, 150], "e4m3", block=block, R=R, cap=500)
        junk = torch.randn((2, 30, 2, 128), device="cuda", dtype=torch.float16)
        for drafts in (30, 1, 17):
            lens = [a.cache.seq_len(i) for i in range(2)]
            packed = [packed_len(n, block, R) for n in lens]
            n = min(drafts, min(p + block + R - 1 - n for p, n in zip(packed, lens)))
            if n <= 0:
                continue
            a.cache.append(junk[:, :n], junk[:, :n])
            a.cache.truncate(lens)
            a.check(q := a.queries(1), a.cache.decode(torch.from_numpy(q).cuda()))
        got = images(a.cache, a.lens, 2)
        want = images(Setup([300, 150], "e4m3", block=block, R=R, cap=500).cache, a.lens, 2)
        assert all(np.array_equal(x, y) for g, w in zip(got, want) for x, y in zip(g, w))


def test_pages_go_round():
    """Released sequences give their pages back; others keep their values."""
    s = Setup([500, 400], "i8", block=32, page=128, cap=512, num_pages=8)
    q = s.queries(1)
    s.cache.release(0)
    assert s.cache.free_pages() == 8 - (packed_len(400, 32, 0) + 127) // 128
    K, V = (torch.from_numpy(x[1:2, :300].copy()).cuda().expand(2, -1, -1, -1).contiguous() for x in (s.K, s.V))
    s.cache.append(K, V, [300, 0])
    s.K[0, :300], s.V[0, :300] = s.K[1, :300], s.V[1, :300]
    s.lens = [300, 400]
    s.check(q, s.cache.decode(torch.from_numpy(q).cuda()))


def test_streams_and_a_captured_call():
    s = Setup([900, 77, 260], "e4m3", gq=4, R=32)
    q = [torch.from_numpy(s.queries(n)).cuda() for n in (1, 5, 40)]
    eager = [s.cache.decode(q[0]), s.cache.chunk(q[1]), s.cache.chunk(q[2]), s.cache.window(q[1], 50, 4)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = [s.cache.decode(q[0], stream=side), s.cache.chunk(q[1], stream=side), s.cache.chunk(q[2], stream=side),
             s.cache.window(q[1], 50, 4, stream=side)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(eager, other))
    out = [torch.empty_like(x) for x in eager]
    with torch.cuda.stream(side):
        s.cache.decode(q[0], out=out[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.cache.decode(q[0], out=out[0])
        s.cache.chunk(q[1], out=out[1])
        s.cache.chunk(q[2], out=out[2])
        s.cache.window(q[1], 50, 4, out=out[3])
    for _ in range(4):
        for x in out:
            x.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, out))
        torch.randn(1000, device="cuda").sum().item()


def test_workspace_is_enough_and_outputs_alone_are_written():
    """The smallest workspace works, one byte less is refused, nothing beside out and workspace changes."""
    s = Setup([3000, 20], "i8", R=16)
    q = torch.from_numpy(s.queries(1)).cuda()
    need = kvq.kvq_workspace_bytes(s.cache.handle)
    buf = torch.full((need + 512,), 0x5A, dtype=torch.uint8, device="cuda")
    out = torch.full((2 * s.hq * 128 + 64,), 7.0, device="cuda")
    before = s.cache.arena.clone()
    kvq.kvq_decode_attention(s.cache.handle, q, out, buf, need)
    torch.cuda.synchronize()
    s.check(q.cpu().numpy(), out[:-64])
    assert (out[-64:] == 7).all() and (buf[need:] == 0x5A).all() and torch.equal(before, s.cache.arena)
    with pytest.raises(KvqError) as e:
        kvq.kvq_decode_attention(s.cache.handle, q, out, buf, 16)
    assert e.value.status == kvq.ERR_CAPACITY


def test_offsets_past_32_bits():
    """A head that begins past 4 GiB of the arena, and tokens past 2^23 of one head's codes."""
    n = 9_000_000
    if torch.cuda.mem_get_info()[0] < 12 << 30:
        pytest.skip("not enough device memory")
    c = BlockCache(1, 2, 2, n, "i8", block_tokens=128)
    g = torch.Generator(device="cuda").manual_seed(1)
    part = 500_000
    for k in range(0, n, part):
        m = min(part, n - k)
        x = torch.randn((1, m, 2, 128), generator=g, device="cuda", dtype=torch.float16)
        c.append(x, -x)
    g = torch.Generator(device="cuda").manual_seed(1)
    for k in range(0, n, part):
        last = torch.randn((1, min(part, n - k), 2, 128), generator=g, device="cuda", dtype=torch.float16)
    p = n // 128 * 128
    rows = last[0, -1000:].cpu().numpy()
    Kd, Vd = c.dequant(0, n - 1000, 1000)
    for h in range(2):
        first = -(-(n - 1000) // 128) * 128 - (n - 1000)  # the first whole block of these tokens
        upto = p - (n - 1000)
        want = quantize_blocks(rows[first:upto, h], "i8", 128)[2].astype(np.float32)
        assert np.array_equal(Kd[first:upto, h].cpu().numpy(), want)
        assert np.array_equal(Vd[first:upto, h].cpu().numpy(), -want)
    # one query that sees the last tokens alone
    q = torch.randn((1, 1, 2, 128), generator=g, device="cuda", dtype=torch.float16)
    out = c.window(q, 500)
    k, v = Kd[-500:].double(), Vd[-500:].double()
    for h in range(2):
        w = torch.softmax(q[0, 0, h].double() @ k[:, h].t() / math.sqrt(128), -1)
        assert float((out[0, 0, h] - w @ v[:, h]).abs().max()) < 1e-5
    # values of opposite keys: attention over everything against its mean by parts
    full = c.decode(q[:, 0])
    assert bool(torch.isfinite(full).all())
