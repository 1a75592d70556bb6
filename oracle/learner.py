"""Test infrastructure (numpy, fp64): the learner's step on what a rollout recorded.

Log-probability, entropy and alternatives of logits rows with their gradient; the clipped objective's gradient;
AdamW with fp32 or 8-bit moments.  Written from the definitions, row by row where that is clearer.

Pins (tests/test_oracle_learner.py): uniform and two-valued rows in closed form; both gradients against central
differences of the forward values; the alternatives against a plain sort; codes that are reproduced exactly by
their own values; the mean of the random rounding; one AdamW step by hand.
"""
from __future__ import annotations

import math
from typing import Optional

import numpy as np

from . import philox

BLOCK = 256


def log_softmax(z: np.ndarray, temperature: float):
    """(log p, p, row is empty, row is undefined) of fp64 logits [R][V].  A row without a finite entry (all -inf) is
    empty; one with NaN or +inf is undefined."""
    bad = np.isnan(z).any(axis=1) | np.isposinf(z).any(axis=1)
    empty = ~bad & np.isneginf(z).all(axis=1)
    zz = np.where((bad | empty)[:, None], 0.0, z)
    s = (zz - zz.max(axis=1, keepdims=True)) / temperature
    e = np.exp(s)
    logp = s - np.log(e.sum(axis=1, keepdims=True))
    return logp, np.exp(logp), empty, bad


def token_logprobs(z: np.ndarray, tokens: np.ndarray, temperature: float, top_k: int = 0):
    """(logprobs, entropy, stats [R][2], top ids, top logprobs) by the definitions in the public header."""
    z = np.asarray(z, dtype=np.float64)
    R, V = z.shape
    logp, p, empty, bad = log_softmax(z, temperature)
    with np.errstate(invalid="ignore"):
        entropy = -np.where(p > 0, p * np.where(p > 0, logp, 0.0), 0.0).sum(axis=1)
    zmax = np.where(np.isnan(z), -np.inf, z).max(axis=1)
    with np.errstate(invalid="ignore"):
        s = (z - np.where(np.isfinite(zmax), zmax, 0.0)[:, None]) / temperature
    logsum = np.log(np.exp(np.where((empty | bad)[:, None], 0.0, s)).sum(axis=1))
    lp = np.zeros(R)
    ids, top = np.full((R, top_k), -1, dtype=np.int32), np.full((R, top_k), -np.inf)
    for r in range(R):
        y = int(tokens[r])
        if empty[r]:
            entropy[r], logsum[r] = 0.0, -np.inf
        if bad[r]:
            entropy[r] = logsum[r] = np.nan
        if y >= V:
            lp[r] = np.nan
        elif y >= 0:
            lp[r] = np.nan if bad[r] else -np.inf if empty[r] else logp[r, y]
        if top_k:
            row = np.where(np.isnan(z[r]), -np.inf, z[r])
            order = np.lexsort((np.arange(V), -row))[:top_k]
            order = [v for v in order if row[v] > -np.inf]
            ids[r, : len(order)] = order
            top[r, : len(order)] = np.nan if bad[r] else logp[r, order]
    return lp, entropy, np.stack([zmax, logsum], axis=1), ids, top


def token_logprobs_backward(z: np.ndarray, tokens: np.ndarray, temperature: float, a: Optional[np.ndarray],
                            b: Optional[np.ndarray]) -> np.ndarray:
    """d (sum_r a_r log p_r[y_r] + b_r H_r) / d z."""
    z = np.asarray(z, dtype=np.float64)
    R, V = z.shape
    logp, p, empty, bad = log_softmax(z, temperature)
    out = np.zeros((R, V))
    for r in range(R):
        y = int(tokens[r])
        ar = float(a[r]) if a is not None and y >= 0 else 0.0
        br = float(b[r]) if b is not None else 0.0
        unknown = y >= V and ar != 0.0                   # scored NaN
        if (empty[r] and not unknown) or (ar == 0.0 and br == 0.0):
            continue
        if bad[r] or unknown:
            out[r] = np.nan
            continue
        plp = np.where(p[r] > 0, p[r] * np.where(p[r] > 0, logp[r], 0.0), 0.0)
        out[r] = -ar * p[r] - br * (plp - p[r] * plp.sum())
        if y < V:
            out[r, y] += ar
    return out / temperature


def grpo_gradient(ln, lo, ls, lr, adv, mask, grad_out, eps_clip: float, C: float, beta: float) -> np.ndarray:
    """d (sum_i grad_out_i J_i) / d ln of the masked mean of w (min(rho A, clip(rho) A) - beta k)."""
    ln, lo, ls = (np.asarray(x, dtype=np.float64) for x in (ln, lo, ls))
    n, T = ln.shape
    out = np.zeros((n, T))
    for i in range(n):
        on = np.ones(T, dtype=bool) if mask is None else np.asarray(mask[i]) != 0
        if not on.any():
            continue
        A = float(adv[i])
        for t in np.nonzero(on)[0]:
            d = ln[i, t] - lo[i, t]
            rho = math.exp(d)
            w = min(math.exp(lo[i, t] - ls[i, t]), C)
            below = math.log1p(-eps_clip) if eps_clip < 1 else -math.inf
            flat = d > math.log1p(eps_clip) if A > 0 else d < below
            g = 0.0 if flat else rho * A
            if lr is not None:
                g += beta * math.expm1(float(lr[i, t]) - ln[i, t])
            out[i, t] = w * g
        out[i] *= (1.0 if grad_out is None else float(grad_out[i])) / on.sum()
    return out


# ---- AdamW ----------------------------------------------------------------------
def avg_values(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    """What int8 first-moment codes of one tensor stand for."""
    q = codes.astype(np.float64) / 127.0
    return np.repeat(scales.astype(np.float64), BLOCK)[: len(codes)] * q * np.abs(q)


def sq_values(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    """What uint8 second-moment codes of one tensor stand for."""
    q = codes.astype(np.float64) / 255.0
    return np.repeat(scales.astype(np.float64), BLOCK)[: len(codes)] * q ** 4


def halves(n: int, tensor: int, step: int, seed: int, moment: int = 0) -> np.ndarray:
    """The 16-bit random number of elements 0..n-1 of tensor `tensor` at `step`: of the second moment's rounding, or
    (moment 1) the first's."""
    out = np.empty((n + 7) // 8 * 8, dtype=np.int64)
    octets = np.arange((n + 7) // 8, dtype=np.uint64)
    words = philox.philox4x32_10(octets & np.uint64(0xFFFFFFFF), octets >> np.uint64(32) | np.uint64(moment << 31), tensor, step,
                                 seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF)
    for j, w in enumerate(words):
        out[2 * j::8] = w & 0xFFFF
        out[2 * j + 1::8] = w >> 16
    return out[:n]


def block_scale(x: np.ndarray) -> np.ndarray:
    """Per block of 256 the largest value as fp32; below the smallest normal number: 0."""
    n = len(x)
    top = np.array([x[i:i + BLOCK].max() for i in range(0, n, BLOCK)], dtype=np.float64).astype(np.float32)
    return np.where(top < np.float32(2.0 ** -126), np.float32(0), top)


def quantise_avg(m: np.ndarray, half: Optional[np.ndarray] = None):
    """(int8 codes, fp32 scales): the nearest code on the companded axis, or, with random numbers, the code below or above
    |m|, the upper where (half + 1/2) / 2^16 is less than |m|'s place between the two."""
    scale = block_scale(np.abs(m))
    wide = np.repeat(scale.astype(np.float64), BLOCK)[: len(m)]
    ratio = np.divide(np.abs(m), wide, out=np.zeros_like(m), where=wide > 0)
    if half is not None:
        low = np.minimum(np.floor(127.0 * np.sqrt(ratio)), 126.0)
        lo, hi = (low / 127.0) ** 2, ((low + 1) / 127.0) ** 2
        return ((low + ((half + 0.5) / 65536.0 * (hi - lo) < ratio - lo)) * np.sign(m)).astype(np.int8), scale
    return (np.rint(127.0 * np.sqrt(ratio)) * np.sign(m)).astype(np.int8), scale


def quantise_sq(v: np.ndarray, half: np.ndarray):
    """(uint8 codes, fp32 scales): the code below or above v, the upper where half / 2^16 is less than v's place
    between the two."""
    scale = block_scale(v)
    wide = np.repeat(scale.astype(np.float64), BLOCK)[: len(v)]
    ratio = np.divide(v, wide, out=np.zeros_like(v), where=wide > 0)
    low = np.minimum(np.floor(255.0 * ratio ** 0.25), 254.0)
    lo, hi = (low / 255.0) ** 4, ((low + 1) / 255.0) ** 4
    code = low + (half / 65536.0 * (hi - lo) < ratio - lo)
    code = np.where(ratio > 0, np.maximum(code, 1), 0)
    return code.astype(np.uint8), scale


def adamw(p, g, m, v, step: int, lr: float, beta1: float, beta2: float, eps: float, weight_decay: float,
          grad_scale: float = 1.0):
    """(p, m, v) after one step, in fp64."""
    p, m, v = (np.asarray(x, dtype=np.float64) for x in (p, m, v))
    g = np.asarray(g, dtype=np.float64) * grad_scale
    m = beta1 * m + (1.0 - beta1) * g
    v = beta2 * v + (1.0 - beta2) * g * g
    m_hat, v_hat = m / (1.0 - beta1 ** step), v / (1.0 - beta2 ** step)
    return p - lr * weight_decay * p - lr * m_hat / (np.sqrt(v_hat) + eps), m, v
