"""Sums of the attention over the cache in 4 bits: the weights that tens of thousands of rows give to a slot, values at the end of their range."""
import math

import numpy as np
import pytest
import torch

import paper_2411_01171_amd as si
from attn_helpers import host, strided
from cache4_helpers import device_cache, random_cache
from gpu_helpers import guarded, guards_intact
from test_gpu_cache4_attn import _check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [40, 64, 128])
@pytest.mark.parametrize("N,group,carried", [(40, 1, False), (1100, 1, True), (9216, 8, False), (50001, 1, True)])
def test_weights_of_many_equal_rows(dtype, d, N, group, carried):
    """All rows are one query, so that a slot receives one number again and again: a running sum that rounds with every row drifts one way.

    The query is 1 in channel 0 and scores are powers of two times a code: exact.  A weight has two exponentials (its own and the sum's) of 2^-22 and
    an exponent's fma, below 2, each; the sum that divides it 40 additions and the division one rounding; log2 e of a score below 1 is off by
    2^-24.  The rows of 16 additions each are collected with at most 2 roundings in all, and their halves and what was there join with 3."""
    cap, rows = 40, N * group
    rng = np.random.default_rng(N)
    groups, room = -(-d // 32), (1, 2, 4, 4)[-(-d // 32) - 1]
    codes, scales = np.zeros((1, 1, cap, 16 * groups), np.uint8), np.full((1, 1, cap, room), 127, np.uint8)
    level = rng.integers(0, 16, cap)  # of channel 0; all 16 codes of a 4-bit value
    codes[0, 0, :, 0] = level
    cache, _ = device_cache((codes, scales, codes, scales), d)
    key = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])[level & 7] * np.where(level & 8, -1.0, 1.0)
    q = np.zeros((1, N, group, d), np.float32)
    q[..., 0] = 1.0
    dq = strided(q, dtype, "rows")
    w_in = rng.random((1, 1, cap)).astype(np.float32) * rows
    buf, w = guarded(torch.empty(1, 1, cap, device="cuda"))
    w.copy_(torch.from_numpy(w_in))
    n = si.si_cache4_attn_workspace_bytes(dq, cache, True)
    ws_buf, ws = guarded(n)
    out = torch.empty_like(dq)
    si.si_cache4_attn_forward(dq, cache, out, ws, scale=0.125, weight_in=w if carried else None, weight_out=w, decay=0.5)
    torch.cuda.synchronize()
    assert guards_intact(buf, w.nbytes) and guards_intact(ws_buf, n)
    p = np.exp(0.125 * key)
    p /= p.sum()
    old = 0.5 * w_in[0, 0].astype(np.float64) if carried else 0.0
    each = 2 * (2.0 ** -22 + 2 * 2.0 ** -24 + 2.0 ** -24) + (40 + 1 + 16 + 2 + 1) * 2.0 ** -24
    assert each < 5e-6
    tol = 1.01 * (each * rows * p + 2 * 2.0 ** -24 * (rows * p + old))
    err = np.abs(host(w)[0, 0] - (rows * p + old))
    assert (err <= tol).all(), float((err / tol).max())
    v = np.zeros(d)
    v[0] = p @ key
    err = np.abs(host(out)[0] - v)  # all rows the same, and right to bf16's two roundings (spread below 6) or float32's
    assert (host(out)[0] == host(out)[0, :1, :1]).all() and err.max() <= (2.0 ** -8 * 1.01 * 12 if dtype == "bf16" else 1e-5 * 6)
    assert math.isfinite(float(w.sum()))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,cap", [(1, 200), (40, 200), (100, 2000), (300, 20000)])
def test_values_of_the_largest_magnitude(dtype, N, cap):
    """Values of 2^88 and scores that rise slowly, so that weights pass the reference maximum by up to its margin: outputs are no infinities."""
    rng = np.random.default_rng(13)
    B, Hk, d = 1, 2, 64
    arrays = [a.copy() for a in random_cache(rng, B, Hk, cap, d)]
    arrays[0][:] = 0
    arrays[0][..., 0] = 4                                    # 2 in channel 0 ...
    arrays[1][..., 0] = 124 + 4 * np.arange(cap) // cap      # ... times 2^-3 .. 2^0
    arrays[2][:], arrays[3][:] = 0x66, 127 + 86              # 4 2^86
    arrays[2][0, 1] = rng.choice(np.array([0x66, 0x6E, 0xE6, 0xEE], np.uint8), arrays[2][0, 1].shape)
    _check(dtype, B, N, cap, Hk, Hk, d, arrays=arrays, q=np.ones((B, N, Hk, d), np.float32), scale=2.5)
