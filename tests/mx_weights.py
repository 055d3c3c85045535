"""Inputs that show the weights of the 4-bit attention one by one: queries with a single element, so that scores are exact, and
values of which position j has column j alone, so that a column is one weight over the sum of all."""
import numpy as np

import mx_reference as ref

LOG2E = 1.4426950408889634


def inputs(B, H_q, H, T, d, n, seed, far=False):
    """Codes and scales of a cache, queries in 64 bits (exact in bf16 and fp16).  n <= d.  far: values of positions lie up to 2^20 apart."""
    assert n <= d
    rng = np.random.default_rng(seed)
    codes, scales = rng.integers(0, 256, size=(B, H, n, d), dtype=np.uint8), rng.integers(126, 128, size=(B, H, n, d // 16), dtype=np.uint8)
    one = np.zeros((B, H, n, d), dtype=np.uint8)
    one[:, :, np.arange(n), np.arange(n)] = rng.integers(1, 8, size=(B, H, n)) + 8 * rng.integers(0, 2, size=(B, H, n))
    codes[..., d // 2:] = ref.pack(one)
    scales[..., d // 32:] = rng.integers(107, 128, size=(B, H, n, 1)) if far else 127
    q = np.zeros((B, H_q, T, d))
    at = rng.integers(0, d, size=(B, H_q, T))
    np.put_along_axis(q, at[..., None], rng.choice([-2.0, 2.0], size=(B, H_q, T, 1)), -1)
    return codes, scales, q


def scores_and_values(codes, scales, q):
    """Scores [B, H_q, T, n], exact, and the values of column j at position j [B, H_q, 1, n], for a scale of 1."""
    k, v = ref.cache_values(codes, scales)
    n, G = k.shape[2], q.shape[1] // k.shape[1]
    k, v = np.repeat(k, G, 1), np.repeat(v, G, 1)
    return q @ k.swapaxes(-1, -2), v[:, :, np.arange(n), np.arange(n)][:, :, None]


def want_and_bound(s, v):
    """Columns 0 .. n - 1 of the output in 64 bits, and what they may be off by.

    Relative to a column, in steps of 2^-24: weights in two parts of 11 bits, cut, 8; exponentials of a weight and of the merges,
    an unit in the last place each, 8; the sum of up to 128 weights, all positive, in 10 additions one after the other, 10; one
    over it, its products and the sums of parts, 10.  Scores: the factor 1.4427 and its product with the score, two roundings, then the
    subtraction of what lies within 15 of the largest; the sum's the same way, where scores near the largest count.  An absolute
    2^-36 of the largest weight, below which weights have no bits."""
    m = s.max(-1, keepdims=True)
    w = np.exp(s - m)
    total = w.sum(-1, keepdims=True)
    want = w / total * v
    score = 2 * np.abs(s) + 2 * np.abs(s).max(-1, keepdims=True) + (m - s) * LOG2E + 30
    return want, np.abs(want) * (36 + score) * 2.0 ** -24 + 2.0 ** -36 * np.abs(v) / total


def columns(s, v, keep):
    """The columns as the kernel computes them, with keep(weights in units that put the largest at 2^12) in the place of its weights."""
    w = np.exp2((s - s.max(-1, keepdims=True)) * LOG2E + 12)
    return keep(w) / w.sum(-1, keepdims=True) * v


def cut(x, bits, lowest=2.0 ** -24):
    """x cut to `bits` significant bits and to multiples of `lowest`, as fp16 parts are."""
    step = np.maximum(np.exp2(np.floor(np.log2(x)) - bits + 1), lowest)
    return np.floor(x / step) * step
