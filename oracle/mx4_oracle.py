"""Plain 64-bit forms of the 4-bit microscaled format, the grouped products and the router (numpy; test infrastructure only).

Written from the definitions: MXFP4 of the OCP Microscaling Formats specification 1.0, with s = max(floor(log2 a) - 2, -127)."""
from __future__ import annotations

import math

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
EVEN = (0, 2, 4, 6)                     # codes whose mantissa bit is zero: ties go there


def groups(K: int) -> int:
    return (K + 127) // 128


def quantize(x):
    """x [rows, K] (finite, infinite or NaN) -> codes uint8 [rows, 64 G], scales uint8 [G, rows, 4]."""
    x = np.asarray(x, np.float64)
    rows, K = x.shape
    G = groups(K)
    p = np.zeros((rows, 128 * G))
    p[:, :K] = x
    blocks = p.reshape(rows, 4 * G, 32)
    bad = ~np.isfinite(blocks).all(-1)
    a = np.abs(np.where(bad[..., None], 0.0, blocks)).max(-1)
    s = np.where(a > 0, np.frexp(a)[1] - 1 - 2, -127)     # frexp: a = m 2^e with m in [0.5, 1), so floor(log2 a) = e - 1
    s = np.maximum(s, -127)
    v = np.abs(np.where(bad[..., None], 0.0, blocks)) / np.ldexp(1.0, s)[..., None]
    d = np.abs(v[..., None] - GRID)
    code = d.argmin(-1)                                    # the first of two at the same distance ...
    up = np.minimum(code + 1, 7)
    tie = np.take_along_axis(d, up[..., None], -1)[..., 0] == np.take_along_axis(d, code[..., None], -1)[..., 0]
    code = np.where(tie & (up != code) & np.isin(up, EVEN), up, code)
    code = np.where(v > 6, 7, code)
    code = np.where(np.signbit(blocks) & ~bad[..., None], code + 8, code).astype(np.uint8).reshape(rows, 128 * G)
    codes = code[:, 0::2] | (code[:, 1::2] << 4)
    scale = np.where(bad, 255, s + 127).astype(np.uint8).reshape(rows, G, 4).transpose(1, 0, 2)
    return np.ascontiguousarray(codes), np.ascontiguousarray(scale)


def values(codes, scales, K=None):
    """What codes and scales stand for, float64 [rows, 128 G] or its first K columns."""
    c = np.stack([codes & 15, codes >> 4], -1).reshape(codes.shape[0], -1)
    v = np.where(c >= 8, -1.0, 1.0) * GRID[c & 7]
    s = scales.transpose(1, 0, 2).reshape(codes.shape[0], -1).astype(np.int64)
    f = np.where(s == 255, np.nan, np.ldexp(1.0, s - 127))
    v = v * np.repeat(f, 32, 1)
    return v if K is None else v[:, :K]


def gelu(y):
    return y * 0.5 * np.vectorize(math.erfc, otypes=[np.float64])(-y / math.sqrt(2.0))


def spans(group_rows, M):
    """(first, last + 1) row of each group: in order, negative numbers as zero, nothing beyond M."""
    out, at = [], 0
    for n in group_rows:
        end = min(M, at + max(int(n), 0))
        out.append((at, end))
        at = end
    return out


def gathered(x, x_rows, M):
    """Rows of x by index; zeros for an index outside."""
    if x_rows is None:
        return x
    out = np.zeros((M, x.shape[1]))
    ok = (x_rows >= 0) & (x_rows < x.shape[0])
    out[ok] = x[x_rows[ok]]
    return out


def grouped(x, w, bias, group_rows, M, x_rows=None):
    """Sums, sums of magnitudes (both [M, N], NaN where a row belongs to no expert) of a grouped product in 64 bits."""
    N = w[0].shape[0]
    y, mag = np.full((M, N), np.nan), np.full((M, N), np.nan)
    rows = gathered(x, x_rows, M)
    for e, (a, b) in enumerate(spans(group_rows, M)):
        y[a:b] = rows[a:b] @ w[e].T + (bias[e] if bias is not None else 0)
        mag[a:b] = np.abs(rows[a:b]) @ np.abs(w[e]).T + (np.abs(bias[e]) if bias is not None else 0)
    return y, mag


def route(logits, k):
    """experts [T, k], gates (64 bits), group_rows, rows, slots."""
    T, E = logits.shape
    l = np.where(np.isnan(logits), -np.inf, logits.astype(np.float64))
    experts = np.stack([sorted(range(E), key=lambda e: (-l[t, e], e))[:k] for t in range(T)]) if T else np.zeros((0, k), int)
    top = np.take_along_axis(l, experts, 1)
    big = float(np.finfo(np.float32).max)
    fin = np.clip(top, -big, big)
    p = np.where(np.isneginf(top), 0.0, np.exp(fin - fin[:, :1]))
    s = p.sum(1, keepdims=True)
    gates = np.where(s > 0, p / np.where(s > 0, s, 1), 0.0)
    flat = experts.reshape(-1)
    order = np.argsort(flat, kind="stable")
    slots = np.empty_like(order)
    slots[order] = np.arange(order.size)
    return experts, gates, np.bincount(flat, minlength=E), order // k, slots.reshape(T, k)
