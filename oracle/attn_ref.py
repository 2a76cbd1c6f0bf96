"""Reference of the operators on heads of video tokens (float64 NumPy): rotary positions on three axes, key blocks chosen
by a score, attention over listed key blocks.

TEST INFRASTRUCTURE ONLY -- see the package docstring.  Definitions as in include/si.h; heads are arrays [B, N, heads, d].
"""
from __future__ import annotations

import math

import numpy as np

F64 = np.float64


def rope_angles_ref(extent, pairs, theta=1e4, origin=(0, 0, 0), step=(1, 1, 1)):
    """Angles [F*H*W, P] of every grid point, raster order."""
    F, H, W = extent
    out = np.empty((F * H * W, sum(pairs)), F64)
    for n in range(F * H * W):
        at = (n // (H * W), n // W % H, n % W)
        col = 0
        for a in range(3):
            for i in range(pairs[a]):
                out[n, col] = (origin[a] + step[a] * at[a]) * theta ** (-i / pairs[a])
                col += 1
    return out


def rms_norm_ref(x, eps, gain=None):
    x = np.asarray(x, F64)
    y = x / np.sqrt((x * x).mean(axis=-1, keepdims=True) + eps)
    return y if gain is None else y * np.asarray(gain, F64)


def rope_ref(x, angles, halves=False, first=0, norm_eps=None, gain=None):
    """Token n of every batch entry turned by angles[first + n]."""
    x = np.asarray(x, F64)
    if norm_eps is not None:
        x = rms_norm_ref(x, norm_eps, gain)
    N, P = x.shape[1], angles.shape[1]
    c, s = (f(angles[first:first + N])[None, :, None, :] for f in (np.cos, np.sin))
    i1 = np.arange(P) if halves else 2 * np.arange(P)
    i2 = i1 + P if halves else i1 + 1
    y = x.copy()
    y[..., i1] = x[..., i1] * c - x[..., i2] * s
    y[..., i2] = x[..., i1] * s + x[..., i2] * c
    return y


def _clamped(length, b, n):
    return n if length is None else min(max(int(length[b]), 0), n)


def block_scores_ref(q, k, q_block, k_block, q_len=None, k_len=None):
    """[B, kv heads, runs, blocks]; NaN where run or block has no token."""
    q, k = np.asarray(q, F64), np.asarray(k, F64)
    B, N, Hq, d = q.shape
    Nk, Hk = k.shape[1], k.shape[2]
    runs, blocks = -(-N // q_block), -(-Nk // k_block)
    out = np.full((B, Hk, runs, blocks), np.nan)
    for b in range(B):
        nq, nk = _clamped(q_len, b, N), _clamped(k_len, b, Nk)
        for h in range(Hk):
            g = Hq // Hk
            for i in range(-(-nq // q_block)):
                qm = q[b, i * q_block:min((i + 1) * q_block, nq), h * g:(h + 1) * g].reshape(-1, d).mean(axis=0)
                for j in range(-(-nk // k_block)):
                    out[b, h, i, j] = qm @ k[b, j * k_block:min((j + 1) * k_block, nk), h].mean(axis=0)
    return out


def pack_blocks_ref(kept):
    """Truth values [.., blocks] -> int32 words, block j in bit j % 32 of word j // 32."""
    kept = np.asarray(kept, bool)
    n = kept.shape[-1]
    pad = np.zeros(kept.shape[:-1] + ((-n) % 32,), bool)
    bits = np.concatenate([kept, pad], axis=-1).reshape(kept.shape[:-1] + (-1, 32)).astype(np.uint64)
    return (bits << np.arange(32, dtype=np.uint64)).sum(axis=-1).astype(np.uint32).view(np.int32)


def select_ref(q, k, q_block, k_block, keep, q_len=None, k_len=None):
    """Truth values [B, kv heads, runs, blocks]: the `keep` best blocks, ties to the lowest, NaN scores as -infinity."""
    B, N = np.shape(q)[:2]
    Nk = np.shape(k)[1]
    s = block_scores_ref(q, k, q_block, k_block, q_len, k_len)
    kept = np.zeros(s.shape, bool)
    for b in range(B):
        runs, blocks = -(-_clamped(q_len, b, N) // q_block), -(-_clamped(k_len, b, Nk) // k_block)
        for h in range(s.shape[1]):
            for i in range(runs):
                row = np.where(np.isnan(s[b, h, i, :blocks]), -np.inf, s[b, h, i, :blocks])
                kept[b, h, i, sorted(range(blocks), key=lambda j: (-row[j], j))[:keep]] = True
    return kept


def sparse_attention_ref(q, k, v, kept, q_block, k_block, scale=None, q_len=None, k_len=None):
    """Returns (out, spread, mass): spread = sum p |v - out|, mass = sum p |v| (p the softmax weights), for error bounds.
    Rows at and behind q_len hold NaN.  kept None: every block."""
    q, k, v = (np.asarray(t, F64) for t in (q, k, v))
    B, N, Hq, d = q.shape
    Nk, Hk = k.shape[1], k.shape[2]
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    out, spread, mass = (np.full(q.shape, np.nan) for _ in range(3))
    for b in range(B):
        nq, nk = _clamped(q_len, b, N), _clamped(k_len, b, Nk)
        for h in range(Hq):
            hk = h // (Hq // Hk)
            for i in range(-(-nq // q_block)):
                rows = slice(i * q_block, min((i + 1) * q_block, nq))
                at = [n for n in range(nk) if kept is None or kept[b, hk, i, n // k_block]]
                if not at:
                    out[b, rows, h], spread[b, rows, h], mass[b, rows, h] = 0.0, 0.0, 0.0
                    continue
                s = q[b, rows, h] @ k[b, at, hk].T * scale
                p = np.exp(s - s.max(axis=-1, keepdims=True))
                p /= p.sum(axis=-1, keepdims=True)
                vs = v[b, at, hk]
                o = p @ vs
                out[b, rows, h] = o
                mass[b, rows, h] = p @ np.abs(vs)
                for n in range(o.shape[0]):
                    spread[b, rows.start + n, h] = p[n] @ np.abs(vs - o[n])
    return out, spread, mass


def block_forward_attn_ref(x, w, hp, ctx, rope=None, q_block=128, k_block=64, keep=0, return_scores=False):
    """Spatial block (block_ref.block_forward_ref) whose self-attention is rotated and / or restricted to selected blocks.

    rope: keyword arguments (extent, pairs and the rest) of rope_angles_ref, and halves, norm_eps, q_gain, k_gain of rope_ref."""
    from .block_ref import (attention_ref, feature_from_tokens_ref, gelu_erf_ref, group_norm_ref, layer_norm_ref,
                            tokens_from_feature_ref)
    W = {k: np.asarray(v, F64) for k, v in w.items()}
    x = np.asarray(x, F64)
    t = tokens_from_feature_ref(group_norm_ref(x, hp.gn_groups, hp.gn_eps, w["gn_g"], w["gn_b"]), "spatial")
    h = t @ W["w_in"] + W["b_in"]
    a = layer_norm_ref(h, W["ln1_g"], W["ln1_b"], hp.ln_eps)
    split = lambda y: y.reshape(y.shape[0], y.shape[1], hp.heads, -1)  # noqa: E731
    q, k, v = (split(a @ W[n]) for n in ("wq", "wk", "wv"))
    if rope is not None:
        turn = {n: rope[n] for n in ("halves", "norm_eps") if n in rope}
        angles = rope_angles_ref(**{n: rope[n] for n in ("extent", "pairs", "theta", "origin", "step") if n in rope})
        q, k = (rope_ref(y, angles, gain=rope.get(g), **turn) for y, g in ((q, "q_gain"), (k, "k_gain")))
    kept = select_ref(q, k, q_block, k_block, keep) if keep else None
    o = sparse_attention_ref(q, k, v, kept, q_block, k_block)[0].reshape(a.shape[0], a.shape[1], -1)
    h = h + o @ W["wo"] + W["bo"]
    a = layer_norm_ref(h, W["ln2_g"], W["ln2_b"], hp.ln_eps)
    c = np.repeat(np.asarray(ctx, F64), x.shape[2], axis=0)
    h = h + attention_ref(a @ W["wq2"], c @ W["wk2"], c @ W["wv2"], hp.heads) @ W["wo2"] + W["bo2"]
    u = layer_norm_ref(h, W["ln3_g"], W["ln3_b"], hp.ln_eps) @ W["w1"] + W["b1"]
    half = u.shape[-1] // 2
    h = h + (u[..., :half] * gelu_erf_ref(u[..., half:])) @ W["w2"] + W["b2"]
    out = x + feature_from_tokens_ref(h @ W["w_out"] + W["b_out"], "spatial", x.shape)
    return (out, block_scores_ref(q, k, q_block, k_block)) if return_scores else out
