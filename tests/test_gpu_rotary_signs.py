"""Signs of zeros in rotated appends: a cos - b sin and a sin + b cos in 64 bits, rounded once,
sign included; no tolerance.
"""
import numpy as np
import pytest

from block_oracle import rotate
from paper_2607_16248_amd import BlockCache, KVCache
from test_gpu_rotary import tables

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("rot,pairs", [(128, False), (128, True), (32, False)])
def test_signs_of_zeros(dtype, rot, pairs):
    """Rows of zeros of both signs and of numbers whose products underflow, first alone and then among others."""
    n = 64
    rng = np.random.default_rng(rot)
    cos, sin = tables(n, rot, seed=3)
    cos[1], sin[1], cos[2], sin[2] = 1.0, 0.0, 0.0, -1.0
    tiny = [0.0, -0.0, 1e-38, -1e-38] if dtype == "bfloat16" else [0.0, -0.0, 2.0 ** -24, -2.0 ** -24]
    cos[32:], sin[32:] = cos[32:] * np.float32(1e-20), sin[32:] * np.float32(1e-20)
    x = rng.choice(tiny, (1, n, 4, 128))
    x[:, 16:32] = np.where(rng.random((1, 16, 4, 128)) < 0.5, x[:, 16:32], rng.standard_normal((1, 16, 4, 128)))
    x[:, 8:16, :, 64:] = -x[:, 8:16, :, :64]
    q = torch.from_numpy(x).cuda().to(getattr(torch, dtype))
    k = q[:, :, :2].contiguous()
    want = rotate(q.double().cpu().numpy()[0], cos, sin, pairs)
    for c in (BlockCache(1, 4, 2, n, "i8", fp16_window=n), KVCache(1, 4, 2, n, [4], [4], fp16_window=n)):
        out = c.append_rotary(q, k, k, torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda(), pairs=pairs)
        got = out.cpu().numpy()[0]
        assert np.array_equal(got.view(np.uint16), want.view(np.uint16)), np.argwhere(got.view(np.uint16) != want.view(np.uint16))[:5]
        for h in range(2):
            image = c.export(0, h)  # (the fp16 tail alone: keys, then values)
            assert np.array_equal(image[:n * 256].view(np.uint16).reshape(n, 128), want[:, h].view(np.uint16))
            assert np.array_equal(image[n * 256:].view(np.uint16).reshape(n, 128), half(k[0, :, h]).view(np.uint16))


def half(x):
    return x.double().cpu().numpy().astype(np.float16)
