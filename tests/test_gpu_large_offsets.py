"""Windows, token sampling and the teacher loss where offsets pass 32 bits: caches whose
regions or pages lie past 4 GiB, rows of logits past 2^31 elements.

Windows: the tolerance of test_gpu_window.py, against 64-bit attention over the cache's
dequantized values (kvq_dequant has its own tests).  Rows: those past the border give
what they give in a call of their own (tokens) or lie where the definition has them.
"""
import math

import numpy as np
import pytest

from paper_2607_16248_amd import kvq

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_distill import check_row  # noqa: E402
from test_gpu_sample import check as check_tokens  # noqa: E402


def check_window(cache, s, n, q, got, window, sinks, gv):
    """q, got [n_q][hq][128] of sequence s of n tokens."""
    n_q, hq = q.shape[:2]
    first = max(0, n - n_q + 1 - window)
    held = min(sinks, first)
    parts = ([cache.dequant(s, 0, held)] if held else []) + [cache.dequant(s, first, n - first)]
    kd, vd = (torch.cat([p[i] for p in parts]).double() for i in range(2))
    at = torch.cat([torch.arange(held, device="cuda"), torch.arange(first, n, device="cuda")])
    pos = torch.arange(n - n_q, n, device="cuda")[:, None]
    hidden = (at > pos) | ((at <= pos - window) & (at >= sinks))
    group = hq // kd.shape[1]
    M = vd.abs().unflatten(-1, (128 // gv, gv)).amax(-1).repeat_interleave(gv, -1)
    worst = 0.0
    for h in range(hq):
        k, v, m = kd[:, h // group], vd[:, h // group], M[:, h // group]
        x = q[:, h].double()
        p = torch.softmax((x @ k.t().contiguous() / math.sqrt(128)).masked_fill(hidden, -math.inf), 1)
        A = (x.abs() @ k.abs().t().contiguous()).max().item() * math.log2(math.e) / math.sqrt(128)
        tol = 2 * math.log(2) * 16 * 2.0 ** -24 * A + 2.0 ** -20
        worst = max(worst, (((got[:, h].double() - p @ v).abs() / (p @ m)).max() / tol).item())
    assert worst <= 1, worst
    return worst


def test_window_of_a_head_past_4_gib():
    n, room = (1 << 21) + 4096 + 5, 1 << 24  # the value scales and the fp16 ring lie past 4 GiB
    g = torch.Generator(device="cuda").manual_seed(12)
    K, V = (torch.randn((1, n, 1, 128), generator=g, device="cuda", dtype=torch.half) for _ in range(2))
    cache = kvq.KVCache(1, 4, 1, room, [8], [8], key_group=32, value_group=32, fp16_window=40)
    cache.append(K, V, [n])
    assert cache.arena.numel() > 1 << 32
    for n_q, window, sinks in ((1, 4096, 4), (5, 100, 70), (70, 3001, 4), (1, 30, 0)):
        q = torch.randn((1, n_q, 4, 128), generator=g, device="cuda", dtype=torch.half)
        check_window(cache, 0, n, q[0], cache.window(q, window, sinks)[0], window, sinks, 32)


@pytest.mark.parametrize("page", [0, 4096])
def test_window_of_a_cache_past_4_gib(page):
    # sequence 0 fills 4.4 GB; sequence 1 lies behind it
    lens, cap = (464 * 4096, 6000), 464 * 4096 + 8192
    g = torch.Generator(device="cuda").manual_seed(13)
    cache = kvq.KVCache(2, 32, 8, cap, [8, 8], [8, 8], key_group=32, value_group=32, fp16_window=32, page_tokens=page)
    assert cache.arena.numel() > 1 << 33
    step = 131072
    for t0 in range(0, lens[0], step):
        n = [min(step, max(0, x - t0)) for x in lens]
        K, V = (torch.randn((2, step, 8, 128), generator=g, device="cuda", dtype=torch.half) for _ in range(2))
        cache.append(K, V, n)
    cache.check()
    for n_q, window, sinks in ((1, 4096, 4), (5, 300, 0), (128, 4096, 40), (600, 500, 4)):
        q = torch.randn((2, n_q, 32, 128), generator=g, device="cuda", dtype=torch.half)
        got = cache.window(q, window, sinks)
        for s in range(2):
            check_window(cache, s, lens[s], q[s], got[s], window, sinks, 32)


def test_rows_past_2_31_logits():
    n, v, k = 17000, 128256, 16
    border = (1 << 31) // v
    rows = [0, border - 1, border, border + 1, n - 1]
    g = torch.Generator(device="cuda").manual_seed(14)
    z = torch.empty((n, v), dtype=torch.bfloat16, device="cuda")
    for r in range(0, n, 1000):
        z[r:r + 1000] = 2.5 * torch.randn((1000, v), generator=g, device="cuda")
    assert z.numel() > 1 << 31
    # tokens
    u = torch.rand((n,), generator=g, device="cuda")
    top_k, top_p = torch.full((n,), 50, dtype=torch.int32, device="cuda"), torch.full((n,), 0.9, device="cuda")
    tokens, logprobs = torch.empty((n,), dtype=torch.int32, device="cuda"), torch.empty((n,), device="cuda")
    ws = torch.empty((kvq.dgap_sample_workspace_bytes(n, v),), dtype=torch.uint8, device="cuda")
    kvq.dgap_sample(z, u, tokens, ws, top_k=top_k, top_p=top_p, logprobs=logprobs)
    few = z[rows].contiguous()
    t2, l2 = torch.empty((len(rows),), dtype=torch.int32, device="cuda"), torch.empty((len(rows),), device="cuda")
    kvq.dgap_sample(few, u[rows].contiguous(), t2, ws, top_k=top_k[:len(rows)], top_p=top_p[:len(rows)], logprobs=l2)
    assert torch.equal(tokens[rows], t2) and torch.equal(logprobs[rows], l2)
    check_tokens(few, u[rows].tolist(), k=[50] * len(rows), p=[0.9] * len(rows))
    # the loss alone, the gradient from its log-sum-exp, and both at once in the logits' place
    teacher = 3 * torch.randn((n, k), generator=g, device="cuda") + 4
    index = torch.randint(0, v, (n, k), generator=g, device="cuda").int()
    loss, lse, grad = torch.empty((n,), device="cuda"), torch.empty((n,), device="cuda"), torch.empty_like(z)
    ws = torch.empty((kvq.dgap_distill_workspace_bytes(n, v),), dtype=torch.uint8, device="cuda")
    host = teacher[rows].cpu().numpy(), index[rows].cpu().numpy()
    kvq.dgap_distill(z, teacher, index, 2.0, loss, ws, lse=lse)
    kvq.dgap_distill_backward(z, teacher, index, 2.0, lse, grad)
    for i, r in enumerate(rows):
        check_row(few[i], host[0][i], host[1][i], 2.0, "bf16", 1.0, loss[r].item(), lse[r].item(), grad[r], backward=True)
    del grad
    kvq.dgap_distill(z, teacher, index, 2.0, loss, ws, lse=lse, grad=z)
    for i, r in enumerate(rows):
        check_row(few[i], host[0][i], host[1][i], 2.0, "bf16", 1.0, loss[r].item(), lse[r].item(), z[r])
    assert bool(torch.isfinite(loss).all()) and np.isfinite(z[::500].float().cpu().numpy()).all()
