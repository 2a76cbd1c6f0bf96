"""Inputs and error bounds for the tests of rotary positions, key-block selection and attention over key blocks."""
from __future__ import annotations

import numpy as np
import torch

import si_workloads as wl
from paper_2411_01171_amd.devio import TORCH_DTYPE

HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}  # of a rounding, relative to the value


def draw(rng, shape, dtype, std=1.0):
    return wl.round_to_storage((rng.standard_normal(shape) * std).astype(np.float32), dtype)


def strided(a: np.ndarray, dtype: str, layout: str):
    """Heads [B,N,H,d] on the GPU as a view in one of the layouts that callers have.  What is not the view's is NaN."""
    B, N, H, d = a.shape
    nan = dict(fill_value=float("nan"), dtype=TORCH_DTYPE[dtype], device="cuda")
    if layout == "rows":           # [B, N, H, d]
        t = torch.full((B, N, H, d), **nan)
    elif layout == "projection":   # the middle of rows three times as wide
        t = torch.full((B, N, 3 * H, d), **nan)[:, :, H:2 * H]
    elif layout == "heads":        # [B, H, N, d]
        t = torch.full((B, H, N, d), **nan).transpose(1, 2)
    elif layout == "tokens":       # [N, B, H, d]
        t = torch.full((N, B, H, d), **nan).transpose(0, 1)
    elif layout == "padded":       # rows with room behind every head and in front of the batch entries
        t = torch.full((B, N + 3, H, d + 8), **nan)[:, 2:2 + N, :, :d]
    else:
        raise ValueError(layout)
    t.copy_(torch.from_numpy(a).to("cuda").to(TORCH_DTYPE[dtype]))
    return t


LAYOUTS = ("rows", "projection", "heads", "tokens", "padded")


def host(t) -> np.ndarray:
    return t.float().cpu().numpy().astype(np.float64)


def lengths(values):
    return None if values is None else torch.tensor(values, dtype=torch.int32, device="cuda")


def attention_bound(q, k, spread, mass, out, dtype, scale, keys):
    """Largest error of an implementation with float32 scores, sums and products.

    Scores: a chain of d products and sums, the scale and the exponent's fma round to float32; each is at most 2^-24 of
    sum |q||k| scale (log2 e of it in the exponent), d + 4 of them.  exp2 is good to 2^-22.  A relative error e of every
    weight moves the output by at most e * spread * (1 + e) / (1 - e).  Sums over the keys: `keys` + 64 roundings of
    2^-24 of sum p |v|, twice (numerator and sum).  bf16: weights are rounded (and summed as rounded), and the output."""
    dots = float(np.max(np.abs(np.asarray(q, np.float64)), initial=0.0)) * float(np.max(np.sum(np.abs(np.asarray(k, np.float64)), axis=-1), initial=0.0)) * scale
    e = (q.shape[-1] + 4) * 2.0 ** -24 * 1.4427 * dots + 2.0 ** -22
    if dtype == "bf16":
        e += HALF_STEP["bf16"]
    assert e < 0.1
    return e * (1 + e) / (1 - e) * spread + 2 * (keys + 64) * 2.0 ** -24 * mass + HALF_STEP[dtype] * 1.01 * np.abs(out) + 1e-37
