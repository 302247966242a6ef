"""Plain 64-bit forms of rotated appends, block-scaled caches, their attention and
adjusted logits (numpy), by the definitions in include/kvq.h and include/dgap.h."""
from __future__ import annotations

import numpy as np

TOP = {"i8": 127.0, "e4m3": 448.0}
# the magnitudes that a type holds, in the order of their codes
GRID = {"i8": np.arange(128, dtype=np.float64),
        "e4m3": np.array([m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10) for e in range(16) for m in range(8)][:127])}


def quantize_blocks(x, kind, block):
    """x fp16 [tokens][128] of one head, tokens a multiple of block: (codes as bytes [tokens][128], scales fp32
    [tokens / block], values in float64 [tokens][128])."""
    grid, codes, scales, values = GRID[kind], [], [], []
    mid = (grid[1:] + grid[:-1]) / 2
    for b in x.astype(np.float64).reshape(-1, block, 128):
        top = np.abs(b).max()
        s = np.float32(top / TOP[kind])  # (a quotient by 127 or 7 * 64 has no 53-bit tie)
        y = np.abs(b) / np.float64(s) if s > 0 else np.zeros_like(b)
        lo, hi = np.searchsorted(mid, y, side="left"), np.searchsorted(mid, y, side="right")
        c = np.where(lo % 2 == 0, lo, hi)
        neg = np.signbit(b)
        codes.append(np.where(neg, -c, c).astype(np.int8).view(np.uint8) if kind == "i8" else (c | (neg << 7)).astype(np.uint8))
        scales.append(s)
        values.append(np.where(neg, -1.0, 1.0) * grid[c] * np.float64(s))
    return (np.concatenate(codes) if codes else np.zeros((0, 128), np.uint8), np.array(scales, np.float32),
            np.concatenate(values) if values else np.zeros((0, 128)))


def packed_len(n, block, window):
    return max(0, n - window) // block * block


def head_image(K, V, tk, tv, block, window, packed=None):
    """The canonical image of a head: K, V fp16 [tokens][128]."""
    p = packed_len(len(K), block, window) if packed is None else packed
    kc, ks, _ = quantize_blocks(K[:p], tk, block)
    vc, vs, _ = quantize_blocks(V[:p], tv, block)
    parts = [kc, ks, vc, vs, K[p:], V[p:]]
    return np.concatenate([np.ascontiguousarray(x).view(np.uint8).reshape(-1) for x in parts])


def zero_signs(image, tk, tv, block, window, n):
    """The image with codes of -0 (e4m3) as those of 0: a sign without a number."""
    p = packed_len(n, block, window)
    image = image.copy()
    for at, kind in ((0, tk), (p * 128 + p // block * 4, tv)):
        if kind == "e4m3":
            part = image[at:at + p * 128]
            part[part == 0x80] = 0
    return image


def cached(K, V, tk, tv, block, window, packed=None):
    """Keys and values of a head as its cache stands for them, float64."""
    p = packed_len(len(K), block, window) if packed is None else packed
    k, v = K.astype(np.float64), V.astype(np.float64)
    k[:p], v[:p] = quantize_blocks(K[:p], tk, block)[2], quantize_blocks(V[:p], tv, block)[2]
    return k, v


def rotate(x, cos, sin, pairs):
    """x [tokens][heads][128], cos and sin fp32 [tokens][rot / 2]: float64, then fp16 in one rounding."""
    y = x.astype(np.float64)
    half = cos.shape[1]
    c, s = cos.astype(np.float64)[:, None], sin.astype(np.float64)[:, None]
    if pairs:
        a, b = y[..., 0:2 * half:2].copy(), y[..., 1:2 * half:2].copy()
        y[..., 0:2 * half:2], y[..., 1:2 * half:2] = a * c - b * s, a * s + b * c
    else:
        a, b = y[..., :half].copy(), y[..., half:2 * half].copy()
        y[..., :half], y[..., half:2 * half] = a * c - b * s, a * s + b * c
    return y.astype(np.float16)


def attention(q, k, v, visible):
    """q [rows][128], k, v [tokens][128] float64, visible [rows][tokens]: (output, softmax-weighted |v| per channel, the
    largest sum |q k| log2(e) / sqrt(128) of a row)."""
    f = np.log2(np.e) / np.sqrt(128.0)
    q = q.astype(np.float64)
    x = np.where(visible, q @ k.T * f, -np.inf)
    w = np.exp2(x - x.max(1, keepdims=True))
    w /= w.sum(1, keepdims=True)
    size = np.where(visible, np.abs(q) @ np.abs(k).T * f, 0.0).max(1)
    return w @ v, w @ np.abs(v), size


def adjust(z, tokens=None, length=None, prompt=None, repetition=None, presence=None, frequency=None, bias_token=None,
           bias=None, mask=None, mask_row=None):
    """Rows of logits, float64 in and out; also the largest magnitude met on the way, per logit."""
    z = np.array(z, dtype=np.float64)
    size = np.where(np.isfinite(z), np.abs(z), 0.0)
    n, vocab = z.shape
    for r in range(n):
        rep = 1.0 if repetition is None else np.float64(repetition[r])
        pre = 0.0 if presence is None else np.float64(presence[r])
        fre = 0.0 if frequency is None else np.float64(frequency[r])
        if not (np.isfinite([rep, pre, fre]).all() and rep > 0):
            z[r] = np.nan
            continue
        if tokens is not None:
            h = tokens.shape[1] if length is None else min(max(int(length[r]), 0), tokens.shape[1])
            p = 0 if prompt is None else int(prompt[r])
            for t in set(int(t) for t in tokens[r, :h] if 0 <= t < vocab):
                z[r, t] = z[r, t] / rep if z[r, t] > 0 else z[r, t] * rep
                size[r, t] = max(size[r, t], abs(z[r, t]) if np.isfinite(z[r, t]) else 0)
            made, count = np.unique([t for i, t in enumerate(tokens[r, :h]) if i >= p and 0 <= t < vocab], return_counts=True)
            for t, c in zip(made.astype(int), count):
                z[r, t] -= fre * c + pre
                size[r, t] += abs(fre * c) + abs(pre)
        if bias_token is not None:
            last = {int(t): np.float64(b) for t, b in zip(bias_token[r], bias[r]) if 0 <= t < vocab}
            for t, b in last.items():
                with np.errstate(invalid="ignore"):
                    z[r, t] = -np.inf if b == -np.inf else z[r, t] + b
                size[r, t] += abs(b) if np.isfinite(b) else 0
        if mask is not None:
            m = r if mask_row is None else int(mask_row[r])
            if 0 <= m < len(mask):
                bits = np.unpackbits(mask[m].view(np.uint8), bitorder="little")[:vocab]
                z[r, bits == 0] = -np.inf
    return z, size
