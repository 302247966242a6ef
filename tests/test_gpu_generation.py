"""The operators of a generation step and of the teacher loss together, as a program
runs them: tokens appended to a packed cache, windowed attention over it, DGAP's
correction of the logits, a token drawn from each row, and afterwards the loss of
the steps' logits against a teacher's.  Every part is held against its 64-bit
oracle on the inputs it got (with the tolerances derived in the parts' own tests),
and a captured step against the eager one, bit by bit, over several replays.
"""
import numpy as np
import pytest

from dgap_inputs import gen_weights
from oracle import dgap as odgap
from paper_2607_16248_amd import kvq

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_distill import check_row as check_loss  # noqa: E402
from test_gpu_sample import check as check_tokens  # noqa: E402
from test_gpu_window import Setup  # noqa: E402

VOCAB, WINDOW, SINKS, K = 5003, 48, 4, 24


class Head:
    """Logits out of an attention output: a weight per vocabulary entry and two of the outputs."""

    def __init__(self, width):
        g = torch.Generator(device="cuda").manual_seed(3)
        self.at = torch.randint(0, width, (2, VOCAB), generator=g, device="cuda")
        self.w = 3 * torch.randn((2, VOCAB), generator=g, device="cuda")

    def __call__(self, out):
        x = out.reshape(out.shape[0], -1)
        return x[:, self.at[0]] * self.w[0] + x[:, self.at[1]] * self.w[1]


class Step:
    """The buffers of one step for `batch` rows, and the step."""

    def __init__(self, cache, head, batch, hq):
        w = gen_weights(1, det_bias=0.0)
        t = [torch.from_numpy(np.ascontiguousarray(x)).cuda() for x in (w.w1, w.b1, w.w2, w.c1, w.cb1, w.c2)]
        self.weights, self.cache, self.head, self.batch = (w, t), cache, head, batch
        self.params = kvq.dgap_params(VOCAB, K, odgap.TAU, t[0], t[1], t[2], w.b2, t[3], t[4], t[5], w.cb2)
        self.q = torch.zeros((batch, 1, hq, 128), dtype=torch.half, device="cuda")
        self.u = torch.zeros((batch,), device="cuda")
        self.tokens = torch.zeros((batch,), dtype=torch.int32, device="cuda")
        self.logprobs = torch.zeros((batch,), device="cuda")
        self.out = torch.zeros((batch, 1, hq, 128), device="cuda")
        self.T = torch.tensor([0.7, 1.0, 1.4][:batch], device="cuda")
        self.k = torch.tensor([40, 0, 200][:batch], dtype=torch.int32, device="cuda")
        self.p = torch.tensor([0.9, 0.95, 1.0][:batch], device="cuda")
        self.teacher = torch.zeros((batch, 32), device="cuda")
        self.index = torch.zeros((batch, 32), dtype=torch.int32, device="cuda")
        self.loss, self.lse = torch.zeros((batch,), device="cuda"), torch.zeros((batch,), device="cuda")
        self.grad = torch.zeros((batch, VOCAB), device="cuda")
        u8 = dict(dtype=torch.uint8, device="cuda")
        self.ws = [torch.empty((kvq.kvq_window_workspace_bytes(cache.handle, 1, WINDOW, SINKS),), **u8),
                   torch.empty((kvq.dgap_workspace_bytes(batch, VOCAB, K),), **u8),
                   torch.empty((kvq.dgap_sample_workspace_bytes(batch, VOCAB),), **u8),
                   torch.empty((kvq.dgap_distill_workspace_bytes(batch, VOCAB),), **u8)]

    def run(self):
        kvq.kvq_window_attention(self.cache.handle, self.q, 1, WINDOW, SINKS, self.out, self.ws[0])
        self.plain = self.head(self.out)
        self.logits = self.plain.clone()
        kvq.dgap_restore(self.params, self.logits, self.batch, self.ws[1])
        kvq.dgap_sample(self.logits, self.u, self.tokens, self.ws[2], temperature=self.T, top_k=self.k, top_p=self.p,
                        logprobs=self.logprobs)
        kvq.dgap_distill(self.plain, self.teacher, self.index, 2.0, self.loss, self.ws[3], lse=self.lse, grad=self.grad)

    def results(self):
        return [x.clone() for x in (self.out, self.logits, self.tokens, self.logprobs, self.loss, self.lse, self.grad)]


@pytest.mark.parametrize("kw", [dict(bk=(2, 4, 8), bv=(2, 4, 1)), dict(bk=2, bv=2, page=64)], ids=["mixed", "paged"])
def test_generation_then_teacher_loss(kw):
    lens = (70, 3, 131)
    c = Setup(lens, R=32, cap=256, **kw)
    head = Head(c.hq * 128)
    s = Step(c.cache, head, 3, c.hq)
    rng = np.random.default_rng(9)
    kept = []
    for step in range(40):
        new = [rng.standard_normal((2, 1, c.hkv, 128)).astype(np.float16) for _ in lens]
        c.kv = [(np.concatenate([k, x[0]]), np.concatenate([v, x[1]])) for (k, v), x in zip(c.kv, new)]
        c.lens = tuple(n + 1 for n in c.lens)
        c.cache.append(torch.from_numpy(np.stack([x[0] for x in new])).cuda(), torch.from_numpy(np.stack([x[1] for x in new])).cuda())
        q, u = c.queries(1), rng.random(3).astype(np.float32)
        s.q.copy_(torch.from_numpy(q))
        s.u.copy_(torch.from_numpy(u))
        t, i = (4 * torch.randn((3, 300), device="cuda") + 6).topk(32)
        s.teacher.copy_(t)
        s.index.copy_(i * 16)
        s.run()
        torch.cuda.synchronize()
        kept.append((s.plain.clone(), s.teacher.clone(), s.index.clone()))
        if step % 8 and step != 39:
            continue
        c.check(q, s.out.cpu().numpy(), WINDOW, SINKS)
        for r in range(3):
            z = s.plain[r].cpu().numpy()
            ref = odgap.restore(z, K, s.weights[0], odgap.TAU)
            same = np.ones(VOCAB, dtype=bool)
            same[ref.idx] = False
            assert np.array_equal(s.logits[r].cpu().numpy()[same], z[same])
        check_tokens(s.logits, list(u), list(s.T.cpu().numpy()), s.k.tolist(), list(s.p.cpu().numpy()))
        want = s.results()
        kvq.dgap_sample(s.logits, s.u, s.tokens, s.ws[2], temperature=s.T, top_k=s.k, top_p=s.p, logprobs=s.logprobs)
        assert (s.tokens == want[2]).all() and (s.logprobs == want[3]).all()
        for r in range(3):
            check_loss(s.plain[r], s.teacher[r].cpu().numpy(), s.index[r].cpu().numpy(), 2.0, "f32", 1.0, s.loss[r].item(),
                       s.lse[r].item(), s.grad[r])
    # the loss of all steps at once, in bf16, and its gradient from the kept log-sum-exp
    z = torch.cat([x[0] for x in kept]).bfloat16()
    t, i = torch.cat([x[1] for x in kept]), torch.cat([x[2] for x in kept])
    n = z.shape[0]
    loss, lse, grad = torch.empty((n,), device="cuda"), torch.empty((n,), device="cuda"), torch.empty_like(z)
    ws = torch.empty((kvq.dgap_distill_workspace_bytes(n, VOCAB),), dtype=torch.uint8, device="cuda")
    kvq.dgap_distill(z, t, i, 2.0, loss, ws, lse=lse)
    scale = torch.full((n,), 1.0 / n, device="cuda")
    kvq.dgap_distill_backward(z, t, i, 2.0, lse, grad, grad_loss=scale)
    for r in range(0, n, 17):
        check_loss(z[r], t[r].cpu().numpy(), i[r].cpu().numpy(), 2.0, "bf16", 1.0 / n, loss[r].item(), lse[r].item(),
                   grad[r], backward=True)


def test_captured_step():
    c = Setup((200, 77, 131), (2, 4, 1), (2, 4, 8), R=32, cap=256)
    head = Head(c.hq * 128)
    s, eager = Step(c.cache, head, 3, c.hq), Step(c.cache, head, 3, c.hq)
    s.run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s.run()
    for n in range(5):
        q, u = torch.from_numpy(c.queries(1)).cuda(), torch.rand((3,), device="cuda")
        t, i = (4 * torch.randn((3, 300), device="cuda") + 6).topk(32)
        for x in (s, eager):
            x.q.copy_(q)
            x.u.copy_(u)
            x.teacher.copy_(t)
            x.index.copy_(i * 16)
        eager.run()
        torch.cuda.synchronize()
        for w in s.ws:  # contents undefined on entry
            w.fill_(0xA5)
        g.replay()
        eager.run()
        torch.cuda.synchronize()
        for a, b in zip(s.results(), eager.results()):
            assert torch.equal(a, b), n
