"""The operators together, as a serving program runs them: a prompt and then tokens
appended with rotation to a block-scaled paged cache, attention over it, drafted
tokens verified and rejected ones dropped, penalties and a grammar's mask on the
logits, a token drawn from each row; every part against its 64-bit oracle on the
inputs it got.
"""
import math

import numpy as np
import pytest

from block_oracle import adjust, attention, cached, packed_len, rotate
from paper_2607_16248_amd import BlockCache, dgap_adjust, dgap_sample, kvq

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

VOCAB, B, HKV, GQ, BLOCK, R = 5003, 3, 2, 4, 32, 48
HQ = HKV * GQ


class Program:
    def __init__(self, types=("e4m3", "i8"), seed=4):
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        self.types = types
        self.cache = BlockCache(B, HQ, HKV, 400, *types, block_tokens=BLOCK, fp16_window=R, page_tokens=64)
        a = np.arange(400)[:, None] * 10000.0 ** (-np.arange(0, 128, 2) / 128)
        self.cos, self.sin = np.cos(a).astype(np.float32), np.sin(a).astype(np.float32)
        self.cd, self.sd = torch.from_numpy(self.cos).cuda(), torch.from_numpy(self.sin).cuda()
        self.K = [np.zeros((0, HKV, 128), np.float16) for _ in range(B)]
        self.V = [np.zeros((0, HKV, 128), np.float16) for _ in range(B)]
        self.packed = [0] * B
        self.weight = torch.randn((HQ * 128, VOCAB), generator=self.g, device="cuda") / 8
        self.history = torch.zeros((B, 64), dtype=torch.int32, device="cuda")
        self.count = [0] * B

    def append(self, n_new):
        n = max(n_new)
        rows = torch.randn((B, n, HQ + 2 * HKV, 128), generator=self.g, device="cuda").bfloat16()
        q, k, v = rows[:, :, :HQ], rows[:, :, HQ:HQ + HKV], rows[:, :, HQ + HKV:]
        out = self.cache.append_rotary(q, k, v, self.cd, self.sd, n_new)
        for s, m in enumerate(n_new):
            at = slice(len(self.K[s]), len(self.K[s]) + m)
            kr, qr = (rotate(x[s, :m].float().cpu().numpy(), self.cos[at], self.sin[at], False) for x in (k, q))
            assert np.array_equal(out[s, :m].cpu().numpy(), qr)
            self.K[s] = np.concatenate([self.K[s], kr])
            self.V[s] = np.concatenate([self.V[s], v[s, :m].float().cpu().numpy().astype(np.float16)])
            self.packed[s] = max(self.packed[s], packed_len(len(self.K[s]), BLOCK, R))
        return out

    def truncate(self, lens):
        self.cache.truncate(lens)
        self.K, self.V = [x[:n] for x, n in zip(self.K, lens)], [x[:n] for x, n in zip(self.V, lens)]

    def check_attention(self, q, out, n):
        q, out = q.cpu().numpy(), out.cpu().numpy().reshape(B, n, HQ, 128)
        for s in range(B):
            L = len(self.K[s])
            vis = np.arange(L) <= np.arange(L - n, L)[:, None]
            for h in range(HKV):
                k, v = cached(self.K[s][:, h], self.V[s][:, h], *self.types, BLOCK, R, packed=self.packed[s])
                for x in range(GQ):
                    ref, mass, size = attention(q[s, :, h * GQ + x], k, v, vis)
                    tol = 2 * math.log(2) * 16 * 2.0 ** -24 * size + 2.0 ** -20
                    assert (np.abs(out[s, :, h * GQ + x] - ref) <= tol[:, None] * mass + 1e-30).all(), (s, h, x)

    def draw(self, out):
        logits = (out.reshape(B, -1) @ self.weight).bfloat16()
        length = torch.tensor(self.count, dtype=torch.int32, device="cuda")
        kw = dict(tokens=self.history, length=length, repetition=torch.full((B,), 1.2, device="cuda"),
                  presence=torch.full((B,), 0.3, device="cuda"), frequency=torch.full((B,), 0.2, device="cuda"),
                  mask=torch.randint(-2 ** 31, 2 ** 31, (B, 157), generator=self.g, device="cuda").int())
        z = torch.empty_like(logits)
        dgap_adjust(logits, z, **kw)
        ref, size = adjust(logits.double().cpu().numpy(), **{k: x.cpu().numpy() for k, x in kw.items()})
        fine = np.isfinite(ref)
        assert np.array_equal(fine, np.isfinite(z.double().cpu().numpy()))
        assert (np.abs(z.double().cpu().numpy() - ref)[fine] <= (5 * 2.0 ** -24 * size + np.abs(np.where(fine, ref, 0)) * 2.0 ** -8)[fine]).all()
        tokens, u = torch.zeros((B,), dtype=torch.int32, device="cuda"), torch.rand((B,), generator=self.g, device="cuda")
        ws = torch.empty(kvq.dgap_sample_workspace_bytes(B, VOCAB), dtype=torch.uint8, device="cuda")
        dgap_sample(z, u, tokens, ws)
        for s, t in enumerate(tokens.tolist()):
            assert 0 <= t < VOCAB and math.isfinite(float(z[s, t]))
            self.history[s, self.count[s]] = t
            self.count[s] += 1


@pytest.mark.parametrize("types", [("e4m3", "i8"), ("i8", "i8")])
def test_a_program(types):
    p = Program(types)
    p.append([70, 5, 130])
    for step in range(12):
        q = p.append([1] * B)
        out = p.cache.decode(q)
        p.check_attention(q, out, 1)
        p.draw(out)
        if step % 4 == 1:  # five drafts, of which some are kept
            held = [len(x) for x in p.K]
            q = p.append([5] * B)
            p.check_attention(q, p.cache.chunk(q), 5)
            p.truncate([max(n + keep, packed) for n, keep, packed in zip(held, (0, 2, 5), p.packed)])
            assert [p.cache.seq_len(s) for s in range(B)] == [len(x) for x in p.K]
        if step == 6:  # a request ends, another takes its place
            p.cache.release(1)
            p.K[1], p.V[1], p.packed[1] = p.K[1][:0], p.V[1][:0], 0
            p.append([0, 90, 0])
    p.cache.check()


def test_captured_attention_and_draw():
    """The device part of a step as one graph (lengths are the host's: one graph per step), replayed with other inputs."""
    p = Program()
    q = p.append([70, 5, 130])[:, :1].contiguous()
    out, z = torch.empty((B, 1, HQ, 128), device="cuda"), torch.empty((B, VOCAB), device="cuda", dtype=torch.bfloat16)
    tokens, u = torch.zeros((B,), dtype=torch.int32, device="cuda"), torch.full((B,), 0.3, device="cuda")
    ws = torch.empty(kvq.dgap_sample_workspace_bytes(B, VOCAB), dtype=torch.uint8, device="cuda")
    pen = torch.full((B,), 1.3, device="cuda")
    part = p.weight[:, :VOCAB].contiguous()

    def step():
        p.cache.decode(q, out=out)
        z.copy_(out.view(B, -1) @ part)
        dgap_adjust(z, tokens=p.history, repetition=pen, presence=pen)
        dgap_sample(z, u, tokens, ws)

    step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):
        q.normal_()
        u.uniform_()
        step()
        want = [x.clone() for x in (out, z, tokens)]
        out.fill_(0)
        tokens.fill_(-7)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (out, z, tokens)))
