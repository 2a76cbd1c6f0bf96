"""Reference of the cache of keys and values in 4 bits (float64 NumPy): what a group of channels is stored as, attention over it with
the weight that every slot received, eviction by that weight.

TEST INFRASTRUCTURE ONLY -- see the package docstring.  Definitions as in include/si.h; heads are arrays [B, N, heads, d],
caches [B, heads, capacity, ..].
"""
from __future__ import annotations

import math

import numpy as np

F64 = np.float64
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def scale_room_ref(d):
    """(groups, bytes of a token's scales)."""
    g = -(-d // 32)
    return g, 4 if g == 3 else g


def encode_group_ref(x):
    """Values of a group (at most 32) -> (codes, scale byte), by trying every scale and every code."""
    x = np.asarray(x, F64)
    if not np.isfinite(x).all():
        return np.zeros(len(x), np.uint8), 255
    most = np.abs(x).max(initial=0.0)
    s = next((s for s in range(2, 253) if most <= 7.0 * 2.0 ** (s - 127)), 252)
    codes = np.empty(len(x), np.uint8)
    for i, v in enumerate(np.abs(x) / 2.0 ** (s - 127)):
        far = np.abs(GRID - v)
        near = np.flatnonzero(far == far.min())  # one, or the two sides of a tie
        codes[i] = near[0] if len(near) == 1 or near[0] % 2 == 0 else near[1]
    return codes | (np.signbit(x).astype(np.uint8) << 3), s


def encode_ref(x):
    """[.., d] -> codes [.., 16 G] and scales [.., S]; scales of a group that does not exist are 0."""
    x = np.asarray(x, F64)
    d = x.shape[-1]
    groups, room = scale_room_ref(d)
    flat = x.reshape(-1, d)
    codes, scales = np.zeros((len(flat), 16 * groups), np.uint8), np.zeros((len(flat), room), np.uint8)
    for n, row in enumerate(flat):
        for g in range(groups):
            c, scales[n, g] = encode_group_ref(row[32 * g:32 * g + 32])
            for i, code in enumerate(c):
                codes[n, 16 * g + i // 2] |= code << (4 * (i % 2))
    return codes.reshape(x.shape[:-1] + (16 * groups,)), scales.reshape(x.shape[:-1] + (room,))


def decode_ref(codes, scales, d):
    """What codes and scales stand for, [.., d]."""
    code = np.stack([codes & 15, codes >> 4], axis=-1).reshape(codes.shape[:-1] + (-1,))[..., :d]
    s = scales[..., np.arange(d) // 32].astype(F64)
    return np.where(code & 8, -1.0, 1.0) * GRID[code & 7] * np.where(s == 255, np.nan, 2.0 ** (s - 127))


def seen_ref(n, q_len, k_len, run):
    """Slots that query n sees: the first so many."""
    if not run:
        return k_len
    return max(0, k_len - q_len + min((n // run + 1) * run, q_len))


def cache_attention_ref(q, k, v, run=0, scale=None, q_len=None, k_len=None, weight_in=None, decay=1.0):
    """k, v [B, heads, capacity, d] as decode_ref gives them.  Returns (out, spread, mass, weight): spread = sum p |v - out|, mass = sum
    p |v|, for error bounds.  Rows at and behind q_len and weights at and behind k_len hold NaN, rows that hold a NaN too: a key's makes all of
    a row NaN, a value's its channel."""
    q, k, v = (np.asarray(t, F64) for t in (q, k, v))
    B, N, Hq, d = q.shape
    Hk, cap = k.shape[1], k.shape[2]
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    out, spread, mass = (np.full(q.shape, np.nan) for _ in range(3))
    weight = np.full((B, Hk, cap), np.nan)
    clamp = lambda length, b, n: n if length is None else min(max(int(length[b]), 0), n)  # noqa: E731
    for b in range(B):
        nq, nk = clamp(q_len, b, N), clamp(k_len, b, cap)
        weight[b, :, :nk] = 0.0 if weight_in is None else decay * np.asarray(weight_in, F64)[b, :, :nk]
        for h in range(Hq):
            hk = h // (Hq // Hk)
            ends = [seen_ref(n, nq, nk, run) for n in range(nq)]
            n = 0
            while n < nq:  # rows that see the same slots
                m = n + 1
                while m < nq and ends[m] == ends[n]:
                    m += 1
                end, rows = ends[n], slice(n, m)
                n = m
                if end == 0:
                    out[b, rows, h], spread[b, rows, h], mass[b, rows, h] = 0.0, 0.0, 0.0
                    continue
                with np.errstate(invalid="ignore"):
                    s = q[b, rows, h] @ k[b, hk, :end].T * scale
                    p = np.exp(s - s.max(axis=-1, keepdims=True))
                    p /= p.sum(axis=-1, keepdims=True)
                    vs = v[b, hk, :end]
                    o = p @ vs
                    out[b, rows, h], mass[b, rows, h] = o, p @ np.abs(vs)
                    for i in range(o.shape[0]):
                        spread[b, rows.start + i, h] = p[i] @ np.abs(vs - o[i])
                weight[b, hk, :end] += p.sum(axis=0)
    return out, spread, mass, weight


def evict_ref(weight, keep, first=0, last=0, k_len=None):
    """Lists [B][heads] of the slots that stay, ascending."""
    weight = np.asarray(weight, F64)
    B, heads, cap = weight.shape
    kept = []
    for b in range(B):
        n = cap if k_len is None else min(max(int(k_len[b]), 0), cap)
        row = []
        for h in range(heads):
            if n <= keep:
                row.append(list(range(n)))
                continue
            w = np.where(np.isnan(weight[b, h]), -np.inf, weight[b, h])
            middle = sorted(range(first, n - last), key=lambda j: (-w[j], j))[:keep - first - last]
            row.append(sorted(list(range(first)) + middle + list(range(n - last, n))))
        kept.append(row)
    return kept
