"""CPU oracle for the cache calls beside LagKV compression -- TEST INFRASTRUCTURE ONLY: attention of a few tokens that
accumulates the weights of the cache rows, eviction by them, and the cache in 8 bits (codes, scales, appending).

Written from the definitions in include/lrsa.h, in 64 bits, for one (sequence, KV head) at a time; shares no code with the HIP path.
"""
from __future__ import annotations

import numpy as np

TOP = {"int8": 127.0, "e4m3": 448.0}
LARGEST = {"int8": 127 * 2.0 ** 121, "e4m3": 240 * 2.0 ** 120}      # values: the next ones are 2^128


def e4m3_value(code: int) -> float:
    """OCP e4m3: sign, 4 bits of exponent (bias 7), 3 bits of fraction; 0x7f and 0xff are no numbers."""
    sign, e, f = -1.0 if code & 0x80 else 1.0, (code >> 3) & 15, code & 7
    if (code & 0x7f) == 0x7f:
        return float("nan")
    return sign * (f / 8 * 2.0 ** -6 if e == 0 else (1 + f / 8) * 2.0 ** (e - 7))


E4M3 = np.array([e4m3_value(c) for c in range(256)])


def decode(codes: np.ndarray, fmt: str) -> np.ndarray:
    """Codes (uint8, or int8 for int8) -> the numbers that they are, without the scale."""
    return codes.view(np.int8).astype(np.float64) if fmt == "int8" else E4M3[codes.view(np.uint8)]


def encode(y: np.ndarray, fmt: str) -> np.ndarray:
    """The nearest code (uint8), ties to the even one."""
    y = np.asarray(y, np.float64)
    if fmt == "int8":
        return np.clip(np.rint(y), -127, 127).astype(np.int8).view(np.uint8)
    mags = E4M3[:127]                                  # ascending, code = index
    a = np.abs(y)
    hi = np.clip(np.searchsorted(mags, a), 0, 126)     # first magnitude >= a
    lo = np.maximum(hi - 1, 0)
    up, down = mags[hi] - a, a - mags[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    code = np.where(mags[hi] == a, hi, code)
    return (code | np.where(np.signbit(y), 0x80, 0)).astype(np.uint8)


def scale_for(top: float, fmt: str) -> float:
    top, s = min(top, LARGEST[fmt]), 2.0 ** -120
    while top > TOP[fmt] * s:
        s *= 2.0
    return s


def append(codes, scales, block, fmt, length, new):
    """codes [cap, d] uint8 and scales [nb] after `new` [count, d] (64 bits) has been appended at `length`; copies."""
    codes, scales, cap = codes.copy(), scales.copy(), len(codes)
    new = new[:max(cap - length, 0)]
    end = length + len(new)
    for j in range(length // block, -(-end // block) if len(new) else 0):
        a, b = max(j * block, length), min((j + 1) * block, end)
        x = np.clip(new[a - length:b - length], -LARGEST[fmt], LARGEST[fmt])
        s = scale_for(np.abs(x).max(), fmt)
        if a > j * block:                              # older rows in front
            old = scales[j]
            s = max(s, old)
            if s > old:
                codes[j * block:a] = encode(decode(codes[j * block:a], fmt) * (old / s), fmt)
        scales[j] = s
        codes[a:b] = encode(x / s, fmt)
    return codes, scales


def values(codes, scales, block, fmt):
    return decode(codes, fmt) * np.repeat(scales.astype(np.float64), block)[:len(codes), None]


def attend(q, K, V, scale=None):
    """q [G, T, d] over K, V [len, d]: token t sees the rows below len - T + 1 + t.  Returns (O [G, T, d], lse [G, T], weight of every
    row, summed over heads and tokens)."""
    q, K, V = (np.asarray(a, np.float64) for a in (q, K, V))
    G, T, d = q.shape
    scale = 1.0 / np.sqrt(d) if scale is None else scale
    O, lse, w_rows = np.zeros((G, T, d)), np.full((G, T), -np.inf), np.zeros(len(K))
    for t in range(T):
        m = len(K) - T + 1 + t
        if m <= 0:
            continue
        s = q[:, t] @ K[:m].T * scale
        top = s.max(1, keepdims=True)
        e = np.exp(s - top)
        z = e.sum(1, keepdims=True)
        O[:, t], lse[:, t] = (e / z) @ V[:m], (top + np.log(z))[:, 0]
        w_rows[:m] += (e / z).sum(0)
    return O, lse, w_rows


def evict_rows(acc, length, sink, recent, budget):
    """The rows that stay, ascending: the first `sink`, the last `recent`, and the largest weights of the others (ties: lowest first)."""
    if length <= budget:
        return np.arange(length)
    middle = list(range(sink, length - recent))
    best = sorted(middle, key=lambda r: (-float(acc[r]), r))[:budget - sink - recent]
    return np.array(list(range(sink)) + sorted(best) + list(range(length - recent, length)), np.int64)


def evict_blocks(x, block, fmt):
    """Values of the rows that stay -> codes and scales of the new cache's blocks."""
    codes, scales = np.zeros(x.shape, np.uint8), np.zeros(-(-len(x) // block))
    for j in range(len(scales)):
        part = x[j * block:(j + 1) * block]
        scales[j] = scale_for(np.abs(part).max(), fmt)
        codes[j * block:(j + 1) * block] = encode(part / scales[j], fmt)
    return codes, scales
