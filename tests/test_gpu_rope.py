"""si_rope_forward against the float64 oracle: every axis split, both pairings, the heads' norm, strides, in place."""
import numpy as np
import pytest
import torch

import oracle
import paper_2411_01171_amd as si
from attn_helpers import HALF_STEP, LAYOUTS, draw, host, strided

pytestmark = pytest.mark.gpu


def _bound(x, y, dtype, normed, d):
    """Products, sum and the sine / cosine (of an angle off by 2^-24 of a revolution, and rounded): 8 half steps of float32 of
    |x1| + |x2|; the norm d + 8 of the value; one rounding of the result."""
    pair = np.abs(x).max(axis=-1, keepdims=True) * 2
    return (8 + 2 * np.pi + (d + 8 if normed else 0)) * 2.0 ** -24 * pair + HALF_STEP[dtype] * 1.01 * np.abs(y) + 1e-37


def _check(dtype, B, N, Hq, Hk, d, extent, pairs, layout="rows", out_layout="rows", halves=False, norm=False, gains=True, first=0,
           origin=(0, 0, 0), step=(1, 1, 1), theta=1e4, in_place=False, seed=0):
    rng = np.random.default_rng(seed)
    q, k = draw(rng, (B, N, Hq, d), dtype), draw(rng, (B, N, Hk, d), dtype)
    gq, gk = draw(rng, (d,), dtype), draw(rng, (d,), dtype)
    dq, dk = strided(q, dtype, layout), strided(k, dtype, layout)
    oq, ok = (dq, dk) if in_place else (strided(np.zeros_like(q), dtype, out_layout), strided(np.zeros_like(k), dtype, out_layout))
    g = [torch.from_numpy(t).to("cuda").to(dq.dtype) if norm and gains else None for t in (gq, gk)]
    rope = si.Rope(extent, pairs, theta=theta, layout=si.SI_ROPE_HALVES if halves else si.SI_ROPE_INTERLEAVED, origin=origin, step=step,
                   norm_eps=1e-6 if norm else None, q_gain=g[0], k_gain=g[1])
    si.si_rope_forward(dq, dk, rope, oq, ok, first=first)
    torch.cuda.synchronize()
    angles = oracle.rope_angles_ref(extent, pairs, theta, origin, step)
    for got, x, gain in ((oq, q, gq), (ok, k, gk)):
        ref = oracle.rope_ref(x, angles, halves, first, 1e-6 if norm else None, gain if norm and gains else None)
        base = oracle.rms_norm_ref(x, 1e-6, gain if gains else None) if norm else np.asarray(x, np.float64)
        assert (np.abs(host(got) - ref) <= _bound(base, ref, dtype, norm, d)).all()
        left = 2 * sum(pairs)
        if not norm:
            assert np.array_equal(host(got)[..., left:], np.asarray(x, np.float64)[..., left:])
    if not in_place:
        assert np.array_equal(host(dq), q) and np.array_equal(host(dk), k)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("d,pairs", [(8, (1, 2, 1)), (40, (6, 7, 7)), (40, (0, 4, 4)), (64, (8, 12, 12)), (80, (13, 10, 13)),
                                     (128, (22, 21, 21)), (128, (64, 0, 0)), (104, (0, 0, 4))])
def test_axes_and_widths(dtype, halves, norm, d, pairs):
    _check(dtype, 2, 3 * 5 * 7, 3, 3, d, (3, 5, 7), pairs, halves=halves, norm=norm)


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("out_layout", LAYOUTS)
def test_strides(layout, out_layout):
    _check("bf16", 2, 33, 4, 4, 64, (3, 1, 11), (8, 12, 12), layout=layout, out_layout=out_layout)
    _check("f32", 2, 33, 4, 4, 40, (1, 3, 11), (0, 4, 4), layout=layout, out_layout=out_layout, halves=True, norm=True)


@pytest.mark.parametrize("halves,norm", [(False, False), (True, True)])
@pytest.mark.parametrize("layout", ["rows", "projection", "heads"])
def test_in_place(layout, halves, norm):
    _check("bf16", 2, 65, 5, 5, 64, (1, 5, 13), (0, 16, 16), layout=layout, in_place=True, halves=halves, norm=norm)


@pytest.mark.parametrize("heads", [(1, 1), (2, 1), (7, 3), (32, 8), (9, 2)])
@pytest.mark.parametrize("norm", [False, True])
def test_heads_shared_by_queries(heads, norm):
    _check("bf16", 1, 20, heads[0], heads[1], 64, (1, 4, 5), (4, 4, 8), norm=norm)


@pytest.mark.parametrize("tokens", [1, 2, 31, 32, 33, 1000])
def test_token_counts_and_windows_of_a_grid(tokens):
    """A window of tokens turns as it does in the whole grid."""
    _check("f32", 1, tokens, 2, 2, 64, (4, 20, 13), (8, 8, 8), first=4 * 20 * 13 - tokens, halves=True)


@pytest.mark.parametrize("origin,step", [((10.0 ** 6, 0, 0), (1, 1, 1)), ((-3.5, 2.0 ** 30, 0.25), (0.5, 1, 0.125)), ((0, 0, 0), (0, -1, 1e5))])
def test_far_and_scaled_positions(origin, step):
    _check("f32", 1, 60, 1, 1, 96, (3, 4, 5), (16, 16, 16), origin=origin, step=step)


def test_gains_are_optional_and_theta_is_free():
    _check("bf16", 1, 12, 2, 2, 64, (1, 3, 4), (0, 16, 16), norm=True, gains=False, theta=256.0)
    _check("f32", 1, 12, 2, 2, 64, (1, 3, 4), (0, 16, 16), theta=0.5)


def test_queries_alone_and_no_tokens():
    x = torch.randn(1, 6, 2, 64, device="cuda")
    rope = si.Rope((1, 2, 3), (0, 8, 8))
    out, both, other = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    si.si_rope_forward(x, None, rope, out, None)
    si.si_rope_forward(x, x.clone(), rope, both, other)
    assert torch.equal(out, both) and torch.equal(out, other)
    none = x[:, :0]
    si.si_rope_forward(none, none, rope, none.clone(), none.clone())


def test_values_that_are_not_finite_stay_in_their_pair():
    x = torch.zeros(1, 2, 1, 64, device="cuda")
    x[0, 1, 0, 3], x[0, 1, 0, 40], x[0, 0, 0, 63] = float("nan"), float("inf"), float("-inf")
    out = torch.empty_like(x)
    si.si_rope_forward(x, None, si.Rope((1, 1, 2), (0, 4, 8)), out, None)
    got = out.cpu()[0, :, 0]
    assert torch.isnan(got[1, 2:4]).all() and got[1, 40] == float("inf") and got[0, 63] == float("-inf")
    rest = got.clone()
    rest[1, 2:4], rest[1, 40], rest[0, 63] = 0, 0, 0
    assert (rest == 0).all()


def test_another_stream_and_a_captured_call():
    x = torch.randn(2, 70, 4, 64, device="cuda", dtype=torch.bfloat16)
    rope = si.Rope((1, 7, 10), (0, 16, 16), norm_eps=1e-6)
    ref, out = torch.empty_like(x), torch.empty_like(x)
    si.si_rope_forward(x, None, rope, ref, None)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    si.si_rope_forward(x, None, rope, out, None, stream=stream)
    stream.synchronize()
    assert torch.equal(out, ref)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        si.si_rope_forward(x, None, rope, out, None)
    for i in range(3):
        x.normal_()
        si.si_rope_forward(x, None, rope, ref, None)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, ref), i


def test_angles_keep_their_digits_in_float32():
    """Pairs (1, 0) and (0, 1) come out as cosines and sines.  Sine and cosine of a float32 angle are good to a step, 2^-24 for
    values up to one; what the angle loses in float32 comes back by one fma, half a step.  Without it the angle alone, rounded
    to 2^-25 of half a turn, would be 1.6 times 2^-24 off."""
    N, d, pairs, theta = 4096, 128, (0, 0, 64), 1e4
    x = torch.zeros(1, N, 2, d, device="cuda")
    x[..., 0, 0::2], x[..., 1, 1::2] = 1.0, 1.0
    out = torch.empty_like(x)
    si.si_rope_forward(x, None, si.Rope((1, 1, N), pairs, theta=theta), out, None)
    angle = oracle.rope_angles_ref((1, 1, N), pairs, theta)
    cos, sin, got = np.cos(angle), np.sin(angle), host(out)[0]
    for have, want in ((got[:, 0, 0::2], cos), (got[:, 0, 1::2], sin), (got[:, 1, 0::2], -sin), (got[:, 1, 1::2], cos)):
        steps = float(np.abs(have - want).max() * 2 ** 24)
        assert steps <= 1.5
