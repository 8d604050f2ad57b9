"""Plain numpy forms of the MX4 operators (microscaled 4-bit floating point).

The format: a block of 32 consecutive channels holds a scale byte b, worth
2^(b-127), and 32 e2m1 codes.  Everything here is written from that definition,
in float64 where nothing is said to be rounded; no code is shared with the
library.
"""
from __future__ import annotations

import math

import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
# the halfway points between levels, each with the level (by code) that a value
# exactly there goes to: the even one
HALFWAY = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
TIE_CODE = np.array([0, 2, 2, 4, 4, 6, 6])


def scale_bytes(v):
    """The scale byte of each block [..., 32] of fp32 values."""
    bits = np.abs(np.ascontiguousarray(v, dtype=np.float32)).view(np.uint32)
    field = (bits.max(-1) >> 23).astype(np.int64)
    return np.where(field == 255, 255, np.maximum(field - 2, 0)).astype(np.uint8)


def codes_of(t):
    """e2m1 codes of values t (float64, already divided by their scale)."""
    a = np.abs(t)
    code = np.searchsorted(HALFWAY, a, side="left")  # halfway points below a
    tie = np.minimum(np.searchsorted(HALFWAY, a, side="left"), len(HALFWAY) - 1)
    code = np.where(a == HALFWAY[tie], TIE_CODE[tie], code)
    return (code | (np.signbit(t) * 8)).astype(np.uint8)


def to_mx4(v):
    """fp32 [rows, K] -> codes [rows, K / 2], scales [ceil(K / 256), rows, 8]."""
    v = np.asarray(v, dtype=np.float32)
    rows, K = v.shape
    blocks = v.reshape(rows, K // 32, 32)
    b = scale_bytes(blocks)
    with np.errstate(invalid="ignore", over="ignore"):
        t = np.ldexp(blocks.astype(np.float64), (127 - b.astype(np.int64))[..., None])
    t[b == 255] = 0.0
    c = codes_of(t).reshape(rows, K)
    tiles = -(-K // 256)
    e = np.zeros((tiles, rows, 8), dtype=np.uint8)
    for i in range(K // 32):
        e[i // 8, :, i % 8] = b[:, i]
    return c[:, 0::2] | (c[:, 1::2] << 4), e


def values(c, e):
    """float64 values of codes and scales."""
    rows, K = c.shape[0], 2 * c.shape[1]
    codes = np.empty((rows, K), dtype=np.int64)
    codes[:, 0::2], codes[:, 1::2] = c & 15, c >> 4
    level = np.where(codes & 8, -1.0, 1.0) * LEVELS[codes & 7]
    b = np.stack([e[i // 8, :, i % 8] for i in range(K // 32)], 1).astype(np.int64)
    v = np.ldexp(level.reshape(rows, -1, 32), (b - 127)[..., None])
    v[b == 255] = np.nan
    return v.reshape(rows, K)


def pack(c, e):
    """Packed weights, index by index."""
    N, K = c.shape[0], 2 * c.shape[1]
    T, B = -(-K // 256), -(-N // 32)
    codes = np.zeros((B, T, 4, 2, 32, 16), dtype=np.uint8)
    scales = np.zeros((T, B, 2, 32, 4), dtype=np.uint8)
    for t in range(T):
        for s in range(4):
            for h in range(2):
                block = 8 * t + 4 * h + s
                if block * 32 >= K:
                    continue
                for b in range(B):
                    n = min(32, N - 32 * b)
                    codes[b, t, s, h, :n] = c[32 * b:32 * b + n, 16 * block:16 * block + 16]
                    scales[t, b, h, :n, s] = e[t, 32 * b:32 * b + n, 4 * h + s]
    return np.concatenate([codes.reshape(-1), scales.reshape(-1)])


def activations(x, z=None, inv_s=None):
    """The fp32 values that ot_quantize_act_mx4 quantizes."""
    v = np.asarray(x).astype(np.float32)
    if z is not None:
        with np.errstate(invalid="ignore", over="ignore"):
            v = (v - z.astype(np.float32)) * inv_s.astype(np.float32)
    return v


def fold(W, b, z, s):
    """(codes, scales, bprime in float64) of ot_fold_weights_mx4."""
    w = W.astype(np.float32)
    c, e = to_mx4(w * s.astype(np.float32) if s is not None else w)
    bias = np.zeros(W.shape[0])
    if z is not None:
        bias = np.array([math.fsum(r) for r in W.astype(np.float64) * z.astype(np.float64)])
    return c, e, bias + (b.astype(np.float64) if b is not None else 0.0)


def linear(x, w, bprime):
    """float64 outputs for float64 values of the operands, before the rounding
    to fp16, and the sum of the magnitudes that enter each."""
    y = x @ w.T + bprime.astype(np.float64)
    return y, np.abs(x) @ np.abs(w).T + np.abs(bprime.astype(np.float64))


def top_k(logits, k):
    """[M, k] experts by falling logit, ties to the lower number, NaN last."""
    l = np.where(np.isnan(logits.astype(np.float64)), -np.inf, logits.astype(np.float64))
    nan = np.isnan(logits.astype(np.float64))
    M, E = l.shape
    return np.array([sorted(range(E), key=lambda j: (bool(nan[m, j]), -l[m, j], j))[:k]
                     for m in range(M)], dtype=np.int64).reshape(M, k)


def moe(x, logits, k, w1, b1, w2, b2, act):
    """float64 outputs of the mixture-of-experts layer: x [M, H], w1 [E, F1, H],
    w2 [E, H, F] as float64 values, b1 [E, F1], b2 [E, H] or None; and the hidden
    activations before their quantization, {(m, j): [F]}."""
    M, H = x.shape
    y, hidden = np.zeros((M, H)), {}
    for m, experts in enumerate(top_k(logits, k)):
        l = logits[m].astype(np.float64)
        experts = [e for e in experts if not np.isnan(l[e]) and l[e] != -np.inf]
        if not experts:
            continue
        most = max(l[e] for e in experts)
        p = np.array([1.0 if l[e] == most else np.exp(l[e] - most) for e in experts])
        p /= p.sum()
        for j, e in enumerate(experts):
            g = w1[e] @ x[m] + (b1[e] if b1 is not None else 0.0)
            F = w2.shape[2]
            h = np.maximum(g, 0) if act == "relu" else g[:F] / (1 + np.exp(-g[:F])) * g[F:]
            hidden[m, j] = h
            q = values(*to_mx4(h[None].astype(np.float32)))[0]
            y[m] += p[j] * (w2[e] @ q + (b2[e] if b2 is not None else 0.0))
    return y, hidden
