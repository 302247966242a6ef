"""dgap_sample where a row's searches end among more elements than its list holds and
far below its largest logit, at u next to 1: the token lies inside the row and where
the 64-bit definition has it.

Border in cumulative mass: within 2^-22 of the total (test_gpu_sample.py derives it:
weights of 24 bits, 2^-23 with the exponential's error, whole sums, and less than
2^-26 of the total left out).  A token is right if its exact share of the mass, from
`before` to `upto`, meets u times the kept total moved by no more than that; with a
top-p below 1 its kept prefix may end 2^-22 of the mass earlier or later, with a
min-p where a weight is within 2^-22 of it.
"""
import math

import numpy as np
import pytest

from paper_2607_16248_amd import kvq

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

EPS = 2.0 ** -22
NEAR_ONE = [1 - 2.0 ** -24, 1 - 2.0 ** -23, 1 - 2.0 ** -20, 0.99999, 1 - 2.0 ** -14, 0.9997, 0.5, 0.0]


def draws(z, u, T=1.0, k=0, p=1.0, m=0.0):
    """Tokens and log-probabilities of one row for every u."""
    n, v = len(u), z.numel()
    rows = z.cuda()[None].expand(n, v).contiguous()
    full = lambda x, t: torch.full((n,), x, dtype=t, device="cuda")  # noqa: E731
    tokens, logprobs = full(-7, torch.int32), full(7.0, torch.float32)
    ws = torch.full((kvq.dgap_sample_workspace_bytes(n, v),), 0xA5, dtype=torch.uint8, device="cuda")
    kvq.dgap_sample(rows, torch.tensor(u, dtype=torch.float32, device="cuda"), tokens, ws, temperature=full(T, torch.float32),
                    top_k=full(k, torch.int32), top_p=full(p, torch.float32), min_p=full(m, torch.float32), logprobs=logprobs)
    torch.cuda.synchronize()
    return tokens.cpu().numpy(), logprobs.cpu().numpy()


def check(z, u, T=1.0, k=0, p=1.0, m=0.0):
    tokens, logprobs = draws(z, u, T, k, p, m)
    T, p, m = (float(np.float32(x)) for x in (T, p, m))
    x = z.double().numpy()
    order = np.argsort(-x, kind="stable")
    w = np.exp((x[order] - x[order[0]]) / T)
    place = np.empty(len(x), dtype=np.int64)
    place[order] = np.arange(len(x))
    n = k if 0 < k < len(x) else len(x)
    upto = np.cumsum(w[:n])
    ends = [n, n]  # fewest and most elements that may be kept
    if p < 1:
        for i, e in enumerate((-EPS, EPS)):
            ends[i] = min(n, int(np.searchsorted(upto, (p + e) * upto[-1], side="left")) + 1)
    if m > 0:
        for i, e in enumerate((EPS, -EPS)):
            ends[i] = max(1, min(ends[i], int((w[:n] >= m * (1 + e)).sum())))
    least, most = upto[ends[0] - 1], upto[ends[1] - 1]
    for token, lp, x in zip(tokens, logprobs, u):
        assert 0 <= token < len(place), (token, x)
        at = place[token]
        assert at < ends[1], (token, x, at, ends)
        before, to = upto[at] - w[at], upto[at]
        x = float(np.float32(x))
        assert before <= (x + EPS) * most and to >= (x - EPS) * least, (token, x, before / most, to / most)
        # (2^-22 for the kept mass, and where it may end)
        want, slack = math.log(w[at] / most), EPS + math.log(most / least)
        assert abs(lp - want) <= slack + 2.0 ** -23 * abs(want), (token, x, lp, want)


def lead(vocab, top, rest, at=7):
    z = rest if torch.is_tensor(rest) else torch.full((vocab,), float(rest))
    z[at] = top
    return z


def noise(vocab, sigma, seed=5):
    return sigma * torch.randn((vocab,), generator=torch.Generator().manual_seed(seed))


@pytest.mark.parametrize("vocab,gap", [(1 << 24, 26.0), (1 << 24, 17.0), (1 << 21, 26.0), (1000000, 22.0), (1 << 19, 24.0),
                                       (128256, 24.0), (40000, 20.0), (5000, 18.0)])
def test_one_leads_equal_logits(vocab, gap):
    z = lead(vocab, gap, 0.0, at=vocab // 3)
    check(z, NEAR_ONE)
    check(z, NEAR_ONE[:4], p=1 - 2.0 ** -24)
    check(z, NEAR_ONE[:4], k=vocab - vocab // 5, p=1 - 2.0 ** -23)
    check(z, NEAR_ONE[:4], m=math.exp(-gap) * 0.99)


@pytest.mark.parametrize("kind", [torch.float32, torch.float16])
def test_one_leads_noise(kind):
    z = lead(1 << 22, 25.0, noise(1 << 22, 2.0)).to(kind)
    check(z, NEAR_ONE)
    check(z, NEAR_ONE[:5], k=3000000, p=0.9999999)
    check(z, NEAR_ONE[:5], m=math.exp(-24.0))
    check(z, NEAR_ONE[:5], T=2.0, k=2000000)


def test_long_top_k_with_a_shorter_nucleus():
    # what lies between the filters' ends is more than a list
    for vocab, sigma in ((128256, 2.5), (1 << 20, 2.0)):
        z = noise(vocab, sigma)
        u = [0.0, 0.1, 0.37, 0.5, 0.9, 0.999, 1 - 2.0 ** -20, 1 - 2.0 ** -24]
        for k, p in ((3000, 0.8), (5000, 0.95), (20000, 0.8), (20000, 0.95)):
            check(z, u, T=0.8, k=k, p=p)
            check(z, u, T=1.2, k=k, p=p, m=0.001)


def test_thousands_an_fp32_step_below_the_leader():
    # a temperature so low that the next fp32 number is many bins away: a range's end takes in what its bins do not hold
    for vocab in (9000, 200000):
        z = torch.full((vocab,), 3.0)
        z[::2] = float(np.nextafter(np.float32(3.0), np.float32(0.0)))
        z[1::2][5000 if vocab > 9000 else 900:] = -1.0
        for T in (1e-6, 2e-8, 1e-30):
            check(z, [0.0, 0.4, 0.999], T=T)
            check(z, [0.0, 0.4, 0.999], T=T, k=vocab // 3, p=0.7)
