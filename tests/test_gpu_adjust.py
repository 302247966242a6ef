"""Adjusted logits on the GPU against 64 bits, through the public call.

A logit takes at most five fp32 roundings (quotient, penalty, two differences, bias) at
the largest magnitude M met on the way: 5 * 2^-24 M, and one of its own type,
finfo.eps / 2 of the result (or half the type's smallest step).
"""
import numpy as np
import pytest

from block_oracle import adjust
from paper_2607_16248_amd import dgap_adjust, dgap_sample, kvq

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def check(z, out, **kw):
    host = {k: None if x is None else x.cpu().numpy() for k, x in kw.items()}
    if host.get("mask") is not None:
        host["mask"] = np.ascontiguousarray(host["mask"])
    ref, size = adjust(z.double().cpu().numpy(), **host)
    got = out.double().cpu().numpy()
    info = torch.finfo(out.dtype)
    top = info.max * (1 + info.eps / 4)
    assert np.array_equal(np.isnan(got), np.isnan(ref))
    fine = np.isfinite(ref) & (np.abs(ref) <= top)
    big = ~fine & ~np.isnan(ref)  # (infinite, or beyond the type)
    assert np.array_equal(got[big], np.copysign(np.inf, ref[big]))
    tol = 5 * 2.0 ** -24 * size + np.abs(np.where(fine, ref, 0)) * info.eps / 2 + info.smallest_normal * info.eps
    err = np.abs(np.where(fine, got - np.where(fine, ref, 0), 0))
    assert (err <= tol).all(), float((err / tol).max())


def settings(n, vocab, history, biases, states, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.rand(s, generator=g, device="cuda")  # noqa: E731
    kw = {}
    if history:
        kw["tokens"] = ((vocab + 3) * rnd(n, history) ** 3).int() - 1  # (a few outside the vocabulary, at both ends)
        kw["length"] = ((history + 3) * rnd(n)).int() - 1              # (negative and too long ones)
        kw["prompt"] = ((history + 2) * rnd(n)).int() - 1
        kw["repetition"] = torch.where(rnd(n) < 0.3, 1.0, 0.7 + rnd(n))
        kw["presence"], kw["frequency"] = rnd(n) - 0.3, rnd(n) - 0.3
    if biases:
        kw["bias_token"] = ((vocab + 2) * rnd(n, biases)).int() - 1    # (the same token twice, too)
        kw["bias"] = 5 * torch.randn((n, biases), generator=g, device="cuda")
    if states:
        words = (vocab + 31) // 32 + 1
        kw["mask"] = torch.randint(-2 ** 31, 2 ** 31, (states, words), generator=g, device="cuda").int()
        kw["mask_row"] = torch.randint(-1, states + 1, (n,), generator=g, device="cuda").int()
    return kw


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("n,vocab,history,biases,states", [
    (1, 1, 3, 2, 1), (2, 31, 1, 0, 0), (5, 4096, 100, 7, 2), (3, 4097, 5000, 0, 3), (4, 8191, 0, 300, 0), (7, 12345, 64, 20, 4),
    (2, 128256, 3000, 16, 2)])
def test_against_64_bits(kind, n, vocab, history, biases, states):
    g = torch.Generator(device="cuda").manual_seed(vocab)
    kw = settings(n, vocab, history, biases, states, n + vocab)
    for width, at in ((vocab, 0), (vocab + 5, 0), (vocab + 8, 3), (vocab + 16, 8)):
        buf = (4 * torch.randn((n * width + 64,), generator=g, device="cuda")).to(TYPES[kind])
        z = buf[at:at + n * width].view(n, width)[:, :vocab]
        out = torch.full((n, vocab + 7), 9.0, device="cuda", dtype=TYPES[kind])
        dgap_adjust(z, out[:, :vocab], **kw)
        check(z, out[:, :vocab], **kw)
        assert (out[:, vocab:] == 9).all()
        same = torch.empty_like(buf)[at:at + n * width].view(n, width)[:, :vocab]  # (aligned as z is)
        dgap_adjust(z, same, **kw)
        assert torch.equal(same.nan_to_num(nan=123.0), out[:, :vocab].nan_to_num(nan=123.0))
        before = buf.clone()
        dgap_adjust(z, **kw)  # in place
        assert torch.equal(z.nan_to_num(nan=123.0), same.nan_to_num(nan=123.0))
        rest = torch.ones_like(buf, dtype=torch.bool)
        rest[at:at + n * width].view(n, width)[:, :vocab] = False
        assert torch.equal(buf[rest], before[rest])


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("biases", [0, 40])
@pytest.mark.parametrize("vocab,shift", [(16384, 0), (16389, 3), (33333, 1)])
def test_many_rows_with_long_histories(kind, biases, vocab, shift):
    n = 520 if vocab <= 16384 else 300
    kw = settings(n, vocab, 4100, biases, 3, vocab + biases)
    g = torch.Generator(device="cuda").manual_seed(vocab + 1)
    width = vocab + 8 - vocab % 8
    buf = (4 * torch.randn((n * width + 8,), generator=g, device="cuda")).to(TYPES[kind])
    z = buf[shift:shift + n * width].view(n, width)[:, :vocab]
    out = torch.empty((n, vocab), device="cuda", dtype=TYPES[kind])
    dgap_adjust(z, out, **kw)
    check(z, out, **kw)
    dgap_adjust(z, **kw)  # in place: runs of 16 bytes
    assert torch.equal(z.nan_to_num(nan=123.0), out.nan_to_num(nan=123.0))


@pytest.mark.parametrize("history", [32767, 32768, 70000])
@pytest.mark.parametrize("prompt", [0, 1, 32768])
def test_one_token_again_and_again(history, prompt):
    n, vocab = 3, 5000
    z = torch.randn((n, vocab), device="cuda")
    one = torch.ones((n,), device="cuda")
    kw = {"tokens": torch.full((n, history), 4097, device="cuda", dtype=torch.int32),
          "length": torch.tensor([history, history - 1, 1], device="cuda", dtype=torch.int32),
          "prompt": torch.full((n,), prompt, device="cuda", dtype=torch.int32), "repetition": 1.5 * one, "presence": 0.25 * one,
          "frequency": 2.0 ** -10 * one, "bias_token": torch.tensor([[4097, 3, 3, 4097]] * n, device="cuda", dtype=torch.int32),
          "bias": torch.tensor([[9.0, 1.0, 2.0, -0.5]] * n, device="cuda")}
    out = torch.empty_like(z)
    dgap_adjust(z, out, **kw)
    check(z, out, **kw)
    assert torch.equal(out[:, 4], z[:, 4]) and torch.equal(out[:, 3], z[:, 3] + 2)


@pytest.mark.parametrize("history", [10, 40000])
def test_the_most_biases(history):
    n, vocab = 2, 6000
    kw = settings(n, vocab, history, 65535, 0, history)
    z = torch.randn((n, vocab), device="cuda").half()
    out = torch.empty_like(z)
    dgap_adjust(z, out, **kw)
    check(z, out, **kw)


def test_nothing_to_adjust_keeps_every_bit():
    x = torch.arange(65536, device="cuda").int().to(torch.int16).view(torch.float16).view(4, -1)  # every fp16 number
    out = torch.zeros_like(x)
    dgap_adjust(x, out)
    assert torch.equal(x.view(torch.int16), out.view(torch.int16))
    one = torch.ones((4,), device="cuda")
    tokens = torch.full((4, 3), -1, device="cuda", dtype=torch.int32)
    dgap_adjust(x, out, tokens=tokens, repetition=one, presence=one, frequency=one)
    assert torch.equal(x.view(torch.int16), out.view(torch.int16))


def test_logits_that_are_not_finite():
    inf, nan = float("inf"), float("nan")
    z = torch.tensor([[inf, -inf, nan, 0.0, -0.0, 3.0, -3.0, 1.0]], device="cuda")
    tokens = torch.tensor([[0, 1, 2, 3, 4, 5, 6]], device="cuda", dtype=torch.int32)
    one = lambda x: torch.tensor([x], device="cuda")  # noqa: E731
    out = torch.empty_like(z)
    dgap_adjust(z, out, tokens=tokens, prompt=torch.tensor([7], device="cuda", dtype=torch.int32), repetition=one(2.0))
    assert out[0, 0] == inf and out[0, 1] == -inf and out[0, 2].isnan() and out[0, 3:].tolist() == [0.0, 0.0, 1.5, -6.0, 1.0]
    at = torch.tensor([[0, 2, 5, 6, 7, 7]], device="cuda", dtype=torch.int32)
    b = torch.tensor([[-inf, -inf, -inf, inf, 4.0, nan]], device="cuda")
    dgap_adjust(z, out, bias_token=at, bias=b)
    assert (out[0, [0, 2, 5]] == -inf).all() and out[0, 6] == inf and out[0, 7].isnan()
    dgap_adjust(z, out, bias_token=at[:, [5, 4]], bias=b[:, [5, 4]])  # the last of two counts
    assert out[0, 7] == 5.0
    mask = torch.zeros((1, 1), device="cuda", dtype=torch.int32)
    dgap_adjust(z, out, bias_token=at, bias=b, mask=mask)
    assert (out == -inf).all()  # a mask goes last, NaN or not


@pytest.mark.parametrize("name,value", [("repetition", 0.0), ("repetition", -1.0), ("repetition", float("nan")), ("repetition", float("inf")),
                                        ("presence", float("nan")), ("presence", float("inf")), ("frequency", float("-inf"))])
def test_bad_settings_spoil_their_row(name, value):
    z = torch.randn((3, 5000), device="cuda").half()
    x = torch.tensor([1.0, value, 1.0], device="cuda")
    out = torch.empty_like(z)
    dgap_adjust(z, out, **{name: x})
    assert out[1].isnan().all() and torch.equal(out[[0, 2]], z[[0, 2]])
    tokens, u = torch.zeros((3,), device="cuda", dtype=torch.int32), torch.full((3,), 0.5, device="cuda")
    ws = torch.empty(kvq.dgap_sample_workspace_bytes(3, 5000), dtype=torch.uint8, device="cuda")
    dgap_sample(out, u, tokens, ws)
    assert tokens[1] == -1 and (tokens[[0, 2]] >= 0).all()


def test_a_mask_that_leaves_nothing_or_one():
    z = torch.randn((2, 40000), device="cuda").bfloat16()
    mask = torch.zeros((2, 1250), device="cuda", dtype=torch.int32)
    mask[1, 777] = 1 << 13
    dgap_adjust(z, mask=mask)
    tokens, u = torch.zeros((2,), device="cuda", dtype=torch.int32), torch.full((2,), 0.9, device="cuda")
    ws = torch.empty(kvq.dgap_sample_workspace_bytes(2, 40000), dtype=torch.uint8, device="cuda")
    dgap_sample(z, u, tokens, ws)
    assert tokens.tolist() == [-1, 777 * 32 + 13]


def test_captured_and_on_another_stream():
    kw = settings(6, 9001, 500, 10, 3, 5)
    z = torch.randn((6, 9001), device="cuda")
    want = torch.empty_like(z)
    dgap_adjust(z, want, **kw)
    side = torch.cuda.Stream()
    out = torch.zeros_like(z)
    torch.cuda.synchronize()
    dgap_adjust(z, out, stream=side, **kw)
    side.synchronize()
    assert torch.equal(out.nan_to_num(), want.nan_to_num())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dgap_adjust(z, out, **kw)
    for k in range(4):
        z.normal_()
        dgap_adjust(z, want, **kw)
        out.fill_(0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.nan_to_num(), want.nan_to_num())


def test_offsets_past_32_bits():
    n, vocab = 150, 1 << 24
    z = torch.empty((n, vocab), device="cuda", dtype=torch.float16)
    z[-1].normal_()
    z[0].normal_()
    tokens = torch.randint(0, vocab, (n, 50), device="cuda", dtype=torch.int32)
    f = torch.full((n,), 0.5, device="cuda")
    first, last = z[:1].clone(), z[-1:].clone()
    dgap_adjust(z, tokens=tokens, frequency=f)
    for row, was, k in ((z[:1], first, 0), (z[-1:], last, n - 1)):
        check(was, row, tokens=tokens[k:k + 1], frequency=f[:1])
