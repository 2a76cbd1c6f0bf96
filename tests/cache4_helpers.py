"""Inputs and error bounds for the tests of the cache in 4 bits."""
from __future__ import annotations

import numpy as np
import torch

import oracle
import paper_2411_01171_amd as si
from attn_helpers import HALF_STEP

NAMES = ("k_codes", "k_scales", "v_codes", "v_scales")


def random_cache(rng, B, heads, cap, d):
    """(codes, scales) of keys and of values: what N(0,1) values would be held as, near enough, drawn directly."""
    groups, room = oracle.scale_room_ref(d)

    def part():
        codes = rng.integers(0, 256, (B, heads, cap, 16 * groups), dtype=np.uint8)
        scales = rng.integers(124, 128, (B, heads, cap, room), dtype=np.uint8)  # values up to 0.75 .. 6
        if d % 32:  # channels past the head
            codes[..., d // 2:] = 0
        return codes, scales

    return (*part(), *part())


def device_cache(arrays, d):
    """A Cache4 of these arrays on the GPU, each in the middle of a larger buffer of 0xFF, and the check that the rest still holds that."""
    wholes, views = [], []
    for a in arrays:
        n, room = a.size, 4096
        whole = torch.full((n + (-n) % 256 + 2 * room,), 0xFF, dtype=torch.uint8, device="cuda")
        view = whole[room:room + n].view(a.shape)
        view.copy_(torch.from_numpy(a).to("cuda"))
        wholes.append((whole, n, room))
        views.append(view)

    def intact():
        return all(bool((w[:r] == 0xFF).all()) and bool((w[r + n:] == 0xFF).all()) for w, n, r in wholes)

    return si.Cache4(*views, d), intact


def values(arrays, d):
    return oracle.decode_ref(arrays[0], arrays[1], d), oracle.decode_ref(arrays[2], arrays[3], d)


def _weight_error(q, k, dtype, scale):
    """Relative error of a softmax weight before its division: the score's roundings and exp2's.

    A chain of d products (float32: 3 d, of three parts each) and sums, the scale and the exponent's fma round to float32, each at most 2^-24
    of sum |q||k| scale, log2 e of it in the exponent; the parts' magnitudes add up to at most 1.01 of the value's.  exp2 is
    good to 2^-22."""
    q, k = np.abs(np.asarray(q, np.float64)), np.abs(np.asarray(k, np.float64))
    dots = float(np.nanmax(q, initial=0.0)) * float(np.nanmax(np.nansum(k, axis=-1), initial=0.0)) * scale
    chain = (3 if dtype == "f32" else 1) * q.shape[-1] + 4
    return chain * 2.0 ** -24 * 1.01 * 1.4427 * dots + 2.0 ** -22


def output_bound(q, k, spread, mass, out, dtype, scale, keys):
    """A relative error e of every weight moves the output by at most e * spread * (1 + e) / (1 - e); sums over the keys: `keys` (float32: three
    parts each) + 64 roundings of 2^-24 of sum p |v|, in numerator and sum.  bf16: weights are rounded (and summed as
    rounded), and the output."""
    e = _weight_error(q, k, dtype, scale) + (HALF_STEP["bf16"] if dtype == "bf16" else 0.0)
    assert e < 0.1
    chain = (3 if dtype == "f32" else 1) * keys + 64
    return e * (1 + e) / (1 - e) * spread + 2 * chain * 2.0 ** -24 * mass + HALF_STEP[dtype] * 1.01 * np.abs(out) + 1e-37


def weight_bound(q, k, received, carried, dtype, scale, keys, rows):
    """A row's weight of a slot has the error of its own exponential and that of the sum that divides it (`keys` + 64 roundings), and the sum over
    `rows` rows rounds once each (+ 32 for the joins); what is carried over is multiplied and added."""
    e = _weight_error(q, k, dtype, scale)
    each = 2 * e * (1 + e) / (1 - e) + (keys + 64 + rows + 32) * 2.0 ** -24 * 1.01
    return each * received + 2 * 2.0 ** -24 * 1.01 * (np.abs(carried) + received) + 1e-37
