"""float32 queries and softmax weights go to the matrix cores as three bf16 parts: inputs whose third parts count, against bounds that a lost one breaks."""
import numpy as np
import pytest
import torch

import paper_2411_01171_amd as si
from attn_helpers import host, strided
from cache4_helpers import device_cache
from gpu_helpers import guarded, guards_intact

pytestmark = pytest.mark.gpu


def _parts(x, n):
    """x (float32) as its first n bf16 parts add up, cut as the kernels cut them."""
    x = np.asarray(x, np.float32)
    rest, total = x.copy(), np.zeros(x.shape)
    for _ in range(n):
        part = (rest.view(np.uint32) & np.uint32(0xFFFF0000)).view(np.float32)
        total += part
        rest = rest - part
    return total


def _run(q, d, N):
    """Two slots, unit vectors 0 and 1 as keys and as values: outputs (p0, p1) and the weights of all rows."""
    groups = -(-d // 32)
    codes, scales = np.zeros((1, 1, 2, 16 * groups), np.uint8), np.full((1, 1, 2, (1, 2, 4, 4)[groups - 1]), 127, np.uint8)
    codes[0, 0, 0, 0], codes[0, 0, 1, 0] = 0x02, 0x20
    cache, _ = device_cache((codes, scales, codes, scales), d)
    dq = strided(q, "f32", "rows")
    out, w = torch.empty_like(dq), torch.zeros(1, 1, 2, device="cuda")
    n = si.si_cache4_attn_workspace_bytes(dq, cache, True)
    buf, ws = guarded(n)
    si.si_cache4_attn_forward(dq, cache, out, ws, scale=1.0, weight_out=w)
    torch.cuda.synchronize()
    assert guards_intact(buf, n)
    return host(out)[0, :, 0], host(w)[0, 0]


def _share(s0, s1):
    return 1 / (1 + np.exp(s1 - s0))


@pytest.mark.parametrize("d", [32, 64, 96, 128])
@pytest.mark.parametrize("N", [1, 16, 30, 33, 97, 300])
def test_queries(d, N):
    """Scores 40 and a little more, exact in float32: channel 0 holds 15 bits behind the first part's.  log2 e is off by two roundings of 2^-24, of a
    difference below 1; an exponential has its fma's rounding (below 2) and 2^-22, the sum and the division one rounding each.  Weights of the rows
    add up one rounding each at most."""
    q = np.zeros((1, N, 1, d), np.float32)
    q[0, :, 0, 0] = 40.25 - 2.0 ** -18 * (1 + np.arange(N) % 8)
    q[0, :, 0, 1] = 40.0
    out, w = _run(q, d, N)
    p = _share(q[0, :, 0, 0].astype(np.float64), 40.0)
    e = 2 * (2.0 ** -22 + 2 * 2.0 ** -24 + 2 * 2.0 ** -24) + 4 * 2.0 ** -24
    lost = _share(_parts(q[0, :, 0, 0], 2), 40.0)
    assert (np.abs(lost - p) > 100 * e * p).all()  # without the third part
    assert (np.abs(out[:, 0] - p) <= e * p).all() and (np.abs(out[:, 1] - (1 - p)) <= e * (1 - p)).all()
    for got, want in zip(w, (p.sum(), (1 - p).sum())):
        assert abs(got - want) <= (e + (N + 8) * 2.0 ** -24) * want
    if N <= 33:
        assert abs(lost.sum() - p.sum()) > 10 * (e + (N + 8) * 2.0 ** -24) * p.sum()


@pytest.mark.parametrize("d", [32, 64, 96, 128])
@pytest.mark.parametrize("N", [16, 30, 33, 97, 300])
def test_weights_of_the_second_product(d, N):
    """Slot 1 has the largest score, 0, and weight 1; slot 0 weights with 24 bits of their own.  Scores are exact, the exponent's fma and log2 e are off
    by 2^-24 of less than 4 each, exp2 by 2^-22; the sum, the reciprocal and its product round once each."""
    q = np.zeros((1, N, 1, d), np.float32)
    q[0, :, 0, 0] = -(1 + np.arange(N) / 512).astype(np.float32)
    out, _ = _run(q, d, N)
    x = np.exp(q[0, :, 0, 0].astype(np.float64))
    p = x / (1 + x)
    e = 2.0 ** -22 + 3 * 4 * 2.0 ** -24 * 0.7 + 4 * 2.0 ** -24
    lost = np.abs(_parts(x.astype(np.float32), 2) / (1 + x) - p)
    assert lost.max() > 4 * e * p.max() and np.median(lost / p) > e  # without the third part
    assert (np.abs(out[:, 0] - p) <= e * p).all()
    assert (np.abs(out[:, 1] - (1 - p)) <= e * (1 - p)).all()
