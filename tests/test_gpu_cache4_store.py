"""si_cache4_store and si_cache4_load against the oracle, bit by bit."""
import numpy as np
import pytest
import torch

import oracle
import paper_2411_01171_amd as si
from attn_helpers import LAYOUTS, draw, host, lengths, strided
from cache4_helpers import device_cache, random_cache, values

pytestmark = pytest.mark.gpu


def _check(dtype, B, N, heads, d, cap, first=None, length=None, layout="rows", k=None, v=None, weight=True, seed=0):
    rng = np.random.default_rng(seed)
    k = draw(rng, (B, N, heads, d), dtype) if k is None else k
    v = draw(rng, (B, N, heads, d), dtype, 30.0) if v is None else v
    before = random_cache(rng, B, heads, cap, d)
    cache, intact = device_cache(before, d)
    w0 = rng.random((B, heads, cap)).astype(np.float32)
    w = torch.from_numpy(w0).to("cuda")
    dk, dv = strided(k, dtype, layout), strided(v, dtype, layout)
    for b in range(B):  # what does not count may hold anything
        if length is not None:
            dk[b, min(max(length[b], 0), N):], dv[b, min(max(length[b], 0), N):] = float("nan"), float("inf")
    si.si_cache4_store(dk, dv, cache, first=lengths(first), length=lengths(length), weight=w if weight else None)
    torch.cuda.synchronize()
    assert intact()
    expected, w_expected = [a.copy() for a in before], w0.copy()
    stored = []
    for b in range(B):
        n = N if length is None else min(max(length[b], 0), N)
        at = 0 if first is None else first[b]
        stored += [(b, i, at + i) for i in range(n) if 0 <= at + i < cap]
    for x, t in enumerate((k, v)):
        codes, scales = oracle.encode_ref(t)
        for b, i, slot in stored:
            expected[2 * x][b, :, slot], expected[2 * x + 1][b, :, slot] = codes[b, i], scales[b, i]
    for b, i, slot in stored:
        if weight:
            w_expected[b, :, slot] = 0
    for got, want in zip(cache.tensors, expected):
        assert bool((got.cpu().numpy() == want).all())
    assert np.array_equal(w.cpu().numpy(), w_expected)

    # and back
    kv = [strided(np.full(k.shape, 7.0, np.float32), dtype, layout) for _ in range(2)]
    si.si_cache4_load(cache, *kv, first=lengths(first), length=lengths(length))
    torch.cuda.synchronize()
    for got, held in zip(kv, values(expected, d)):
        want = np.full(k.shape, 7.0)
        for b, i, slot in stored:
            want[b, i] = held[b, :, slot]
        assert np.array_equal(host(got), want, equal_nan=True)
    return cache


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", range(8, 129, 8))
def test_head_widths(dtype, d):
    _check(dtype, 2, 37, 3, d, 50, first=[3, 13])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", LAYOUTS)
def test_strides(dtype, layout):
    _check(dtype, 2, 19, 2, 64, 30, first=[0, 11], layout=layout)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [40, 64, 96, 128])
@pytest.mark.parametrize("N", [1, 2, 63, 64, 65, 130])
def test_lengths_from_one_token_on(dtype, d, N):
    _check(dtype, 1, N, 1, d, N, weight=N % 2 == 0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_padded_batches_and_slots_outside_the_cache(dtype):
    _check(dtype, 4, 20, 2, 64, 25, first=[5, 0, 24, -7], length=[20, 0, 3, 20])
    _check(dtype, 3, 20, 2, 80, 25, first=[6, -100, 25], length=[99, 20, -3])
    _check(dtype, 2, 20, 1, 8, 9, first=[2 ** 31 - 1, -2 ** 31], length=[20, 20])
    _check(dtype, 1, 20, 1, 8, 9)


def test_every_rounding():
    """Ties, values next to them and at the ends of the range, in groups of every magnitude."""
    edges = np.array([0.0, 0.25, 0.5, 0.75, 1.0, 1.25, 1.5, 1.75, 2.0, 2.5, 3.0, 3.5, 4.0, 5.0, 6.0, 6.5, 7.0])
    rows = []
    for e in (-126, -125, -124, -60, -1, 0, 1, 60, 124, 125):
        for top in (3.5000002, 3.75, 4.0, 5.0, 6.0, 6.9999995, 7.0):
            x = np.concatenate([[top], -edges[1:16], np.nextafter(edges[1:9].astype(np.float32), np.float32(9)), -np.nextafter(edges[1:9].astype(np.float32), np.float32(0))])
            rows.append(np.clip(x, -top, top) * 2.0 ** e)
    x = np.array(rows, dtype=np.float32).reshape(1, len(rows), 1, 32)
    assert np.isfinite(x).all()
    _check("f32", 1, len(rows), 1, 32, len(rows), k=x, v=-x)
    x = draw(np.random.default_rng(0), x.shape, "bf16") * 0 + torch.from_numpy(x).to(torch.bfloat16).float().numpy()
    _check("bf16", 1, len(rows), 1, 32, len(rows), k=x, v=-x)


def test_ends_of_the_range():
    x = np.zeros((1, 6, 1, 40), np.float32)
    x[0, 0, 0, :4] = [3.4e38, -3.3e38, 1e38, -1e30]     # above what a bf16 of six times a power of two reaches
    x[0, 1, 0, 39] = 2.0 ** -149                          # subnormal
    x[0, 2, 0, :3] = [1e-38, -2e-38, 0.0]
    x[0, 3, 0, 0] = -0.0
    x[0, 4, 0, :2] = [2.0 ** -126, -2.0 ** -125]
    x[0, 5, 0, 38] = 1.0
    _check("f32", 1, 6, 1, 40, 6, k=x, v=x[:, ::-1].copy())
    held = torch.from_numpy(x).to(torch.bfloat16).float().numpy()
    held[0, 0, 0, 0] = 3.3e38
    held = torch.from_numpy(held).to(torch.bfloat16).float().numpy()
    assert np.isfinite(held).all()
    _check("bf16", 1, 6, 1, 40, 6, k=held, v=held[:, ::-1].copy())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
def test_groups_that_are_not_finite_read_as_nan(dtype, bad):
    rng = np.random.default_rng(3)
    k, v = draw(rng, (1, 9, 2, 80), dtype), draw(rng, (1, 9, 2, 80), dtype)
    k[0, 2, 1, 5] = bad
    v[0, 8, 0, 79] = bad
    _check(dtype, 1, 9, 2, 80, 9, k=k, v=v)


def test_what_every_code_stands_for():
    """All codes under all scales that are written, by both loads."""
    codes = np.arange(256, dtype=np.uint8).reshape(16, 16)
    scales = np.array([2, 3, 100, 126, 127, 128, 200, 251, 252, 255], np.uint8)
    n = len(scales) * 16
    arrays = (np.tile(codes, (len(scales), 1)).reshape(1, 1, n, 16), np.repeat(scales, 16).reshape(1, 1, n, 1))
    cache, _ = device_cache((*arrays, *arrays), 32)
    want = oracle.decode_ref(*arrays, 32).transpose(0, 2, 1, 3)
    for dtype in (torch.bfloat16, torch.float32):
        k, v = torch.empty(1, n, 1, 32, device="cuda", dtype=dtype), torch.empty(1, n, 1, 32, device="cuda", dtype=dtype)
        si.si_cache4_load(cache, k, v)
        assert np.array_equal(host(k), want, equal_nan=True) and np.array_equal(host(v), want, equal_nan=True)


def test_empty_calls():
    cache = si.Cache4.empty(2, 3, 0, 64)
    x = torch.full((2, 5, 3, 64), 7.0, device="cuda")
    si.si_cache4_store(x, x.clone(), cache)
    si.si_cache4_load(cache, x, x.clone())
    full = si.Cache4.empty(2, 3, 4, 64)
    si.si_cache4_store(x[:, :0], x[:, :0], full)
    torch.cuda.synchronize()
    assert (x == 7).all()


def test_offsets_beyond_32_bits():
    """Slots whose codes lie more than 4 GiB behind the first."""
    cap, d = 36_000_000, 128
    cache = si.Cache4(*(torch.zeros(1, 2, cap, n, dtype=torch.uint8, device="cuda") for n in (64, 4, 64, 4)), d)
    rng = np.random.default_rng(4)
    k, v = draw(rng, (1, 5, 2, d), "bf16"), draw(rng, (1, 5, 2, d), "bf16")
    at = lengths([cap - 5])
    weight = torch.ones(1, 2, cap, device="cuda")
    si.si_cache4_store(strided(k, "bf16", "rows"), strided(v, "bf16", "rows"), cache, first=at, weight=weight)
    for x, t in enumerate((k, v)):
        codes, scales = oracle.encode_ref(t)
        for got, want in zip(cache.tensors[2 * x:], (codes, scales)):
            assert np.array_equal(got[:, :, -5:].cpu().numpy(), want.transpose(0, 2, 1, 3))
            assert int(torch.count_nonzero(got[:, :, :-5])) == 0
    assert (weight[:, :, -5:] == 0).all() and (weight[:, :, :-5] == 1).all()
    out = [torch.empty(1, 5, 2, d, device="cuda") for _ in range(2)]
    si.si_cache4_load(cache, *out, first=at)
    for got, t in zip(out, (k, v)):
        assert np.array_equal(host(got), oracle.decode_ref(*oracle.encode_ref(t), d))
