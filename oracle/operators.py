"""Plain 64-bit definitions of the products with 4-bit weights and of the rules on logits, written
from their formulas with numpy, and how far 32-bit kernels may be from them.  Inputs are numpy arrays:
float values as they are stored, widened to float64; codes uint8."""
from __future__ import annotations

import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0])
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}      # of one rounding, relative


def unpack(codes: np.ndarray) -> np.ndarray:
    """[N,K/2] bytes to [N,K] codes: column 2j in the low half of byte j."""
    out = np.empty((codes.shape[0], codes.shape[1] * 2), dtype=np.uint8)
    out[:, 0::2] = codes & 15
    out[:, 1::2] = codes >> 4
    return out


def w4_weights(codes, scales, zeros, group: int, kind: str) -> np.ndarray:
    n = unpack(codes)
    column = np.arange(n.shape[1]) // group
    if kind == "e2m1":
        value = E2M1[n]
    else:
        value = n.astype(np.float64) - (8.0 if zeros is None else zeros.astype(np.float64)[:, column])
    return value * scales.astype(np.float64)[:, column]


def activate(y, act: str):
    if act == "silu":
        with np.errstate(over="ignore"):
            return y / (1.0 + np.exp(-y))
    return np.maximum(y, 0.0) if act == "relu" else y


def matvec_w4(x, codes, scales, zeros=None, group=128, kind="int", bias=None, residual=None, act="identity"):
    """y[m,n] = act(sum_j x[m,j] w[n,j] + bias[n]) + residual[m,n]."""
    y = x.astype(np.float64) @ w4_weights(codes, scales, zeros, group, kind).T
    if bias is not None:
        y = y + bias.astype(np.float64)
    y = activate(y, act)
    return y if residual is None else y + residual.astype(np.float64)


def matvec_w4_bound(x, codes, scales, zeros=None, group=128, kind="int", bias=None, residual=None, act="identity",
                    out="f32"):
    """Largest error of fp32 sums in any order, by arithmetic.  The terms of a group are exact, and
    the integer codes' carry an offset: |16 + code| |x| and (16 + zero) |x|.  A sum of n terms with
    each addition rounded to fp32 is off by at most n 2^-24 times the sum of their absolute values (to
    first order); a term meets the additions of its own group (its columns, and as many again for the
    offsets), of the groups, and of 64 partial sums, and each scaling is another rounding.  Bias,
    activation and residual add a few roundings of the values they work on (the activations' slopes
    are below 1.1; eight roundings cover exp and the division)."""
    K = x.shape[1]
    column = np.arange(K) // group
    n = unpack(codes)
    if kind == "e2m1":
        size = np.abs(E2M1[n])
    else:
        z = 8.0 if zeros is None else zeros.astype(np.float64)[:, column]
        size = (16.0 + n) + (16.0 + z)
    total = np.abs(x.astype(np.float64)) @ (size * np.abs(scales.astype(np.float64)[:, column])).T
    err = (2 * min(group, K) + -(-K // group) + 64 + 4) * 2.0 ** -24 * total
    y = x.astype(np.float64) @ w4_weights(codes, scales, zeros, group, kind).T
    if bias is not None:
        y = y + bias.astype(np.float64)
        err = err + 2.0 ** -24 * (np.abs(y) + err)
    if act != "identity":
        err = 1.1 * err + 8 * 2.0 ** -24 * np.abs(y)
        y = activate(y, act)
    if residual is not None:
        y = y + residual.astype(np.float64)
        err = err + 2.0 ** -24 * (np.abs(y) + err)
    return err + HALF_STEP[out] * (np.abs(y) + err) + (2.0 ** -25 if out == "f16" else 0.0)   # fp16's subnormals


def _cut(a, b, n):
    return slice(max(int(a), 0), max(0, min(int(b), n)))


def logit_rules(z, history=None, ranges=None, penalties=None, bias_ids=None, bias_values=None, bias_ranges=None,
                mask=None):
    """(z', err): the logits under their rules in float64, and how far values rounded to fp32 after each
    operation may be from them (half a step of every intermediate value, amplified by what follows)."""
    z = z.astype(np.float64).copy()
    M, V = z.shape
    err = np.zeros_like(z)
    half = 2.0 ** -24
    with np.errstate(invalid="ignore"):
        for m in range(M):
            if ranges is not None:
                a, b, c, d = (int(v) for v in ranges[m])
                rep, freq, pres = (float(v) for v in penalties[m])
                prompt, output = history[_cut(a, b, len(history))], history[_cut(c, d, len(history))]
                seen = np.zeros(V, dtype=bool)
                count = np.zeros(V)
                for v in prompt:
                    if 0 <= v < V:
                        seen[v] = True
                for v in output:
                    if 0 <= v < V:
                        seen[v] = True
                        count[v] += 1
                for v in np.flatnonzero(seen):
                    z[m, v] = z[m, v] / rep if z[m, v] > 0 else z[m, v] * rep
                    err[m, v] += half * abs(z[m, v])
                    if count[v]:
                        z[m, v] -= count[v] * freq
                        err[m, v] += half * (abs(count[v] * freq) + abs(z[m, v]))
                        z[m, v] -= pres
                        err[m, v] += half * abs(z[m, v])
            if bias_ranges is not None:
                s = _cut(*bias_ranges[m], len(bias_ids))
                last = {int(v): float(w) for v, w in zip(bias_ids[s], bias_values[s])}
                for v, w in last.items():
                    if 0 <= v < V:
                        z[m, v] += w
                        err[m, v] += half * abs(z[m, v])
            if mask is not None:
                ids = np.arange(V)
                word = mask[m].astype(np.int64)[ids // 32] & 0xFFFFFFFF
                z[m, (word >> (ids % 32)) & 1 == 0] = -np.inf
    err[~np.isfinite(z)] = 0.0
    return z, 1.001 * err                       # (the roundings of the errors themselves)


def topk_logprob(z, k):
    """(ids, log-probabilities) of the k best per row of z (float64, -inf and NaN no candidates); (-1, -inf)
    behind the last one, equal values by lower id."""
    M, V = z.shape
    ids = np.full((M, k), -1, dtype=np.int32)
    logp = np.full((M, k), -np.inf)
    for m in range(M):
        real = np.flatnonzero(z[m] > -np.inf)
        if real.size == 0:
            continue
        order = real[np.lexsort((real, -z[m, real]))][:k]
        top = z[m, real].max()
        ids[m, :order.size] = order
        # (not z - (top + log): beside a value of 1e38 the logarithm is nothing)
        logp[m, :order.size] = (z[m, order] - top) - np.log(np.exp(z[m, real] - top).sum())
    return ids, logp
