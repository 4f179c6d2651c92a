"""Plain 64-bit definitions of a drafter's attention (norms and rotation of heads, the cache of 4-bit
floats, attention over it and over prompts), written from their formulas with numpy, and how far kernels
with 32-bit sums may be from them.  Inputs are numpy arrays: float values as they are stored, widened to
float64; codes and scales uint8."""
from __future__ import annotations

import numpy as np

from oracle.operators import E2M1, HALF_STEP, unpack

SMALLEST = {"f32": 2.0 ** -150, "bf16": 2.0 ** -134, "f16": 2.0 ** -25}       # half the step of subnormal values
LARGEST_UNIT = {"f32": 125, "bf16": 125, "f16": 13}                           # exponents: 6 units stay finite


def rounding(value, dtype):
    """Largest error of one rounding of these values to the storage type."""
    return np.maximum(np.abs(value) * HALF_STEP[dtype], SMALLEST[dtype])


# ---------------------------------------------------------------- norms and rotation
def norm_rope(x, positions=None, inv_freq=None, weight=None, eps=1e-6, interleaved=False):
    """x [T,heads,D] with each head's norm and its pairs turned by positions[t] * inv_freq[i]."""
    y = x.astype(np.float64).copy()
    if weight is not None:
        y = y / np.sqrt((y * y).mean(axis=-1, keepdims=True) + eps) * weight.astype(np.float64)
    if inv_freq is not None:
        half = len(inv_freq)
        a = np.arange(0, 2 * half, 2) if interleaved else np.arange(half)
        b = a + 1 if interleaved else a + half
        angle = (positions.astype(np.float64)[:, None] * inv_freq.astype(np.float64))[:, None]
        ya, yb = y[..., a].copy(), y[..., b].copy()
        y[..., a] = ya * np.cos(angle) - yb * np.sin(angle)
        y[..., b] = yb * np.cos(angle) + ya * np.sin(angle)
    return y


def norm_rope_bound(x, positions=None, inv_freq=None, weight=None, eps=1e-6, interleaved=False, dtype="f32"):
    """The mean is a sum of positive terms: 8 in a chain and at most 5 additions across lanes, so off by 13
    roundings at most, half of that after the root; root, division and two products add four more: below
    16 half steps of fp32.  A turn's fraction is off by 2^-51 of the angle, its rounding to fp32 and the
    sine by at most 8 half steps; products and sum add three.  So 27, taken as 32, of each of a pair's two values."""
    y = np.abs(norm_rope(x, None, None, weight, eps))
    off = 32 * 2.0 ** -24 * y
    if inv_freq is not None:
        half = len(inv_freq)
        a = np.arange(0, 2 * half, 2) if interleaved else np.arange(half)
        b = a + 1 if interleaved else a + half
        angle = np.abs(positions.astype(np.float64)[:, None] * inv_freq.astype(np.float64))[:, None]
        pair = (32 * 2.0 ** -24 + angle * 2.0 ** -51) * (y[..., a] + y[..., b])
        off[..., a] = off[..., b] = pair
    want = norm_rope(x, positions, inv_freq, weight, eps, interleaved)
    return off + rounding(np.abs(want) + off, dtype)


# ---------------------------------------------------------------- the cache of 4-bit floats
def kv4_quantise(x, dtype):
    """x [..., D] as (codes [..., D/2], scales [..., D/32]) bytes, by the distances to the fifteen values."""
    blocks = x.astype(np.float64).reshape(*x.shape[:-1], -1, 32)
    top = np.abs(blocks).max(axis=-1)
    e = np.full(top.shape, -126)
    some = top > 0
    with np.errstate(divide="ignore"):
        e[some] = np.frexp(np.where(np.isinf(top[some]), 1.0, top[some]))[1] - 3      # floor(log2) - 2
    e = np.where(top > 7 * np.exp2(e.astype(np.float64)), e + 1, e)
    e = np.where(np.isinf(top), LARGEST_UNIT[dtype], np.clip(e, -126, LARGEST_UNIT[dtype]))
    unit = np.exp2(e.astype(np.float64))[..., None]
    with np.errstate(invalid="ignore"):
        size = np.minimum(np.abs(blocks) / unit, 6.0)
    off = np.abs(size[..., None] - E2M1[:8])
    best = off.min(axis=-1, keepdims=True)
    code = np.where(off == best, np.arange(8) % 2 * 8 + np.arange(8), 99).argmin(axis=-1)    # ties: the even code
    code = (code + 8 * np.signbit(blocks)).reshape(x.shape).astype(np.uint8)
    return code[..., 0::2] | code[..., 1::2] << 4, (e + 127).astype(np.uint8)


def kv4_values(codes, scales, dtype="f32"):
    """What is held, as calls of this type read it."""
    code = unpack(codes.reshape(-1, codes.shape[-1])).reshape(*codes.shape[:-1], -1)
    unit = np.exp2(np.minimum(scales.astype(np.float64), 127 + LARGEST_UNIT[dtype]) - 127)
    return (E2M1[code].reshape(*scales.shape, 32) * unit[..., None]).reshape(code.shape)


def kv4_tokens(codes, scales, page_table, length, dtype="f32"):
    """One sequence's tokens [length, kv_heads, D], and which of them lie in a page of the cache."""
    page_size = codes.shape[2]
    if length == 0:
        return np.zeros((0, codes.shape[1], codes.shape[3] * 2)), np.zeros(0, bool)
    at = np.arange(length)
    page = np.asarray(page_table)[at // page_size]
    held = (page >= 0) & (page < codes.shape[0])
    page = np.where(held, page, 0)
    return kv4_values(codes[page, :, at % page_size], scales[page, :, at % page_size], dtype), held


# ---------------------------------------------------------------- attention
def attention(q, k, v, seen, scale):
    """q [n,heads,D], k and v [m,kv_heads,D], seen [n,m]: (out, sum p |v|, root of sum p^2 v^2, largest bound
    of a score's error by fp32 sums, sum |v| over the keys seen), the last four for the bounds."""
    n, heads, D = q.shape
    group = heads // k.shape[1]
    out, mean, spread, size_v = (np.zeros(q.shape) for _ in range(4))
    score_off = np.zeros((n, heads))
    for h in range(heads):
        kk, vv = k[:, h // group], v[:, h // group]
        with np.errstate(invalid="ignore"):
            s = np.where(seen, q[:, h] @ kk.T * scale, -np.inf)
            size = np.where(seen, np.abs(q[:, h]) @ np.abs(kk).T * abs(scale), 0.0)
        some = seen.any(axis=1)
        if not some.any():
            continue
        top = s[some].max(axis=1, keepdims=True)
        p = np.exp(s[some] - top)
        p /= p.sum(axis=1, keepdims=True)
        with np.errstate(invalid="ignore"):
            clean = np.where(seen[some].any(axis=0)[:, None], vv, 0.0)
            out[some, h] = p @ clean
            mean[some, h] = p @ np.abs(clean)
            spread[some, h] = np.sqrt((p * p) @ (clean * clean))
            size_v[some, h] = seen[some].astype(np.float64) @ np.abs(clean)
        # a sum of D products, and the roundings of scaled score and reference
        score_off[some, h] = ((D + 4) * 2.0 ** -24 * size[some]).max(axis=1) + 4 * 2.0 ** -24 * np.abs(top[:, 0])
    return out, mean, spread, score_off, size_v


WEIGHT_STEP = {"f32": 2.0 ** -23, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}       # of a weight's rounding in the second product

SMALLEST_WEIGHT = {"f32": 2.0 ** -126, "bf16": 2.0 ** -126, "f16": 2.0 ** -32}


def attention_bound(out, mean, spread, score_off, size_v, keys, dtype):
    """Largest error: a weight is off by e^(twice a score's error) - 1, the exponential (4 half steps) and its
    rounding, the sums over keys by a rounding each, and the result is divided and rounded.  Weights are kept
    relative to a reference at most as large as the row's largest (their sum is then 1 or more); fp32 and bf16
    end at 2^-126, where the exponential and the products give zero, so each key's weight may be off by that much
    too.  fp16 weights have normal numbers from 2^-14 on and subnormal ones in steps of 2^-24, relative to a
    reference at least 2^7 below the row's largest: off by half a step, 2^-32 of it."""
    part = 2.2 * score_off[..., None] + WEIGHT_STEP[dtype] + (2 * keys + 16) * 2.0 ** -24
    off = part * (mean + np.abs(out)) + SMALLEST_WEIGHT[dtype] * size_v
    return off + rounding(np.abs(out) + off, dtype)


def attention_norm_bound(out, mean, spread, score_off, size_v, dtype):
    """What the 2-norm of the error over many values may come to: roundings of weights and results have
    independent signs, so the norm of their largest sizes is above the errors' by a root of three.  Sums in fp32
    add 4e-6 of the mean (64 half steps, of which random signs leave a tenth), and scores a tenth of their
    largest error likewise: one of a few hundred is rounded to steps of 2^-16 by its size alone, which moves its
    weight by as much."""
    return HALF_STEP[dtype] * np.linalg.norm(out) + WEIGHT_STEP[dtype] * np.linalg.norm(spread) + \
        np.linalg.norm((4e-6 + 0.1 * score_off[..., None]) * mean) + SMALLEST_WEIGHT[dtype] * np.linalg.norm(size_v)
