"""si_cache4_attn_forward against the float64 oracle, element by element, within a bound derived from its roundings."""
import math

import numpy as np
import pytest
import torch

import oracle
import paper_2411_01171_amd as si
from attn_helpers import LAYOUTS, draw, host, lengths, strided
from cache4_helpers import device_cache, output_bound, random_cache, values, weight_bound
from gpu_helpers import guarded, guards_intact

pytestmark = pytest.mark.gpu


def _forward(q, cache, out, run=0, stream=None, **kw):
    n = si.si_cache4_attn_workspace_bytes(q, cache, weights=kw.get("weight_out") is not None)
    assert n > 0
    buf, ws = guarded(n)
    si.si_cache4_attn_forward(q, cache, out, ws, run=run, stream=stream, **kw)
    torch.cuda.synchronize()
    assert guards_intact(buf, n)


def _check(dtype, B, N, cap, Hq, Hk, d, run=0, q_len=None, k_len=None, layout="rows", out_layout="rows", scale=None, std=1.0, weights=True, seed=0,
           arrays=None, q=None, carried=True):
    rng = np.random.default_rng(seed)
    q = draw(rng, (B, N, Hq, d), dtype, std) if q is None else q
    arrays = random_cache(rng, B, Hk, cap, d) if arrays is None else arrays
    w_in = rng.random((B, Hk, cap)).astype(np.float32)
    k, v = values(arrays, d)
    sent = [a.copy() for a in arrays]
    dq = strided(q, dtype, layout)
    for b in range(B):  # what does not count may hold anything
        if q_len is not None:
            dq[b, min(max(q_len[b], 0), N):] = float("nan")
        if k_len is not None:
            for a, fill in zip(sent, (0xFF, 0xFF, 0x77, 0xFF)):
                a[b, :, min(max(k_len[b], 0), cap):] = fill
            w_in[b, :, min(max(k_len[b], 0), cap):] = np.nan
    cache, intact = device_cache(sent, d)
    out = strided(np.full(q.shape, 7.0, np.float32), dtype, out_layout)
    kw = {}
    if weights:
        buf, w_out = guarded(torch.empty(B, Hk, cap, device="cuda"))
        w_out.fill_(5.0)
        kw = {"weight_out": w_out, "decay": 0.75}
        if carried:
            kw["weight_in"] = torch.from_numpy(w_in).to("cuda")
    _forward(dq, cache, out, run, scale=scale, q_len=lengths(q_len), k_len=lengths(k_len), **kw)
    assert intact()
    sc = 1 / math.sqrt(d) if scale is None else scale
    ref, spread, mass, w_ref = oracle.cache_attention_ref(q, k, v, run, sc, q_len, k_len, w_in if carried else None, 0.75)
    got, left = host(out), np.isnan(ref)
    assert (got[left] == 7.0).all()  # rows behind the lengths stay
    tol = output_bound(q, k, spread, mass, ref, dtype, sc, cap)
    err = np.abs(got - ref)
    assert (err[~left] <= tol[~left]).all(), float(np.max(err[~left] / tol[~left]))
    if weights:
        assert guards_intact(buf, w_out.nbytes)
        w_got, left = host(w_out), np.isnan(w_ref)
        assert (w_got[left] == 5.0).all()
        old = np.where(left, 0.0, 0.75 * np.nan_to_num(w_in) if carried else 0.0)
        tol = weight_bound(q, k, np.maximum(w_ref - old, 0), old, dtype, sc, cap, N * (Hq // Hk))
        err = np.abs(w_got - w_ref)
        assert (err[~left] <= tol[~left]).all(), float(np.max(err[~left] / tol[~left]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", range(8, 129, 8))
def test_head_widths(dtype, d):
    _check(dtype, 1, 5, 333, 2, 2, d)
    _check(dtype, 1, 130, 200, 2, 2, d)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [32, 64, 96, 128])
@pytest.mark.parametrize("N", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 257, 300])
def test_numbers_of_queries(dtype, d, N):
    _check(dtype, 1, N, 190, 1, 1, d, weights=N % 2 == 1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [1, 70, 200])
@pytest.mark.parametrize("keys", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 95, 96, 97, 127, 128, 129, 255, 256, 257, 1000])
def test_key_counts(dtype, N, keys):
    _check(dtype, 1, N, keys, 1, 1, 64)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads", [(2, 1), (8, 2), (7, 1), (32, 2), (48, 1)])
@pytest.mark.parametrize("N", [1, 3, 40])
def test_heads_shared_by_queries(dtype, heads, N):
    _check(dtype, 2, N, 300, heads[0], heads[1], 64)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("out_layout", LAYOUTS)
def test_strides(dtype, layout, out_layout):
    _check(dtype, 2, 50, 150, 3, 3, 64, layout=layout, out_layout=out_layout)
    _check(dtype, 2, 140, 150, 3, 3, 128, layout=layout, out_layout=out_layout)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [5, 200])
@pytest.mark.parametrize("run", [0, 1, 33])
@pytest.mark.parametrize("q_len,k_len", [([0, 150, 200], [640, 0, 1]), ([1, 64, 65], [64, 65, 63]), ([-3, 999, 128], [7000, -1, 610])])
def test_padded_batches(dtype, N, run, q_len, k_len):
    """Fewer slots than queries among them: with runs their first rows see nothing."""
    _check(dtype, 3, N, 650, 2, 1, 64, run=run, q_len=q_len, k_len=k_len)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [40, 128])
@pytest.mark.parametrize("run", [1, 2, 5, 16, 31, 32, 33, 64, 100, 127, 128, 129, 160, 400])
@pytest.mark.parametrize("group", [1, 4])
def test_runs(dtype, d, run, group):
    _check(dtype, 1, 161, 300, group, 1, d, run=run)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("run", [0, 1, 7])
def test_more_queries_than_slots(dtype, run):
    _check(dtype, 2, 90, 20, 2, 2, 64, run=run)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,group,run", [(1, 1, 0), (1, 4, 0), (8, 4, 1), (40, 2, 0), (300, 1, 0)])
@pytest.mark.parametrize("cap", [5000, 70001])
def test_long_caches(dtype, N, group, run, cap):
    """A tile's keys are dealt out to several workgroups and joined."""
    _check(dtype, 1, N, cap, 2 * group, 2, 64 if N > 8 else 128, run=run)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [1e-3, 0.5])
@pytest.mark.parametrize("N", [4, 140])
def test_flat_and_peaked_weights(dtype, scale, N):
    """Scores up to some tens: the reference maximum rises many times on the way."""
    _check(dtype, 1, N, 1500, 1, 1, 64, scale=scale)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [3, 40, 150])
@pytest.mark.parametrize("sign", [1, -1])
def test_rising_and_falling_scores(dtype, N, sign):
    d, cap = 64, 64 * 12
    rng = np.random.default_rng(2)
    arrays = [a.copy() for a in random_cache(rng, 1, 1, cap, d)]
    arrays[0][:] = 0
    arrays[0][..., 0] = 4 if sign > 0 else 12          # 2 or -2 in channel 0 ...
    arrays[1][..., 0] = 124 + np.arange(cap) // 128    # ... times 2^-3 .. 2^2
    _check(dtype, 1, N, cap, 1, 1, d, arrays=arrays, q=np.ones((1, N, 1, d), np.float32), scale=5.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,run", [(6, 0), (6, 1), (150, 0), (150, 1), (150, 50)])
@pytest.mark.parametrize("which", ["key", "value", "query"])
def test_not_finite_shows_where_it_is_seen_and_nowhere_else(dtype, N, run, which):
    rng = np.random.default_rng(11)
    d, cap = 96, 400
    q = draw(rng, (1, N, 2, d), dtype)
    arrays = [a.copy() for a in random_cache(rng, 1, 2, cap, d)]
    at = cap - N + 2 if N < 20 else cap - N + 60  # among the new tokens
    if which == "key":
        arrays[1][0, 1, at, 2] = 255
    elif which == "value":
        arrays[3][0, 1, at, 1] = 255
    else:
        q[0, 3, 1, 7] = np.nan
    cache, _ = device_cache(arrays, d)
    out = strided(np.zeros(q.shape, np.float32), dtype, "rows")
    w = torch.zeros(1, 2, cap, device="cuda")
    _forward(strided(q, dtype, "rows"), cache, out, run, weight_out=w)
    k, v = values(arrays, d)
    ref, _, _, w_ref = oracle.cache_attention_ref(q, k, v, run)
    assert np.isnan(ref).any() and not np.isnan(ref).all()
    assert np.array_equal(np.isnan(host(out)), np.isnan(ref))
    assert np.array_equal(np.isnan(host(w)), np.isnan(w_ref))
    clean = [a.copy() for a in arrays]
    clean[1][clean[1] == 255], clean[3][clean[3] == 255] = 126, 126
    k, v = values(clean, d)
    ref2, spread, mass, _ = oracle.cache_attention_ref(np.nan_to_num(q), k, v, run)
    ok = ~np.isnan(ref)
    tol = output_bound(np.nan_to_num(q), k, spread, mass, ref2, dtype, 1 / math.sqrt(d), cap)
    if which != "value":  # rows that do not see it are those of the clean cache
        assert (np.abs(host(out) - ref2)[ok] <= tol[ok]).all()
    else:
        assert (np.abs(host(out) - np.where(ok, ref2, 0))[ok] <= tol[ok]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [2, 150])
def test_infinite_queries(dtype, N):
    """+inf among a row's scores makes it NaN; scores of -inf weigh nothing."""
    d, cap = 32, 100
    q = np.zeros((1, N, 1, d), np.float32)
    q[0, :, 0, 0] = -np.inf
    q[0, 1, 0, 0] = np.inf
    arrays = [np.zeros((1, 1, cap, n), np.uint8) for n in (16, 1, 16, 1)]
    arrays[0][:] = 0x22                                   # ones everywhere: no zero meets the infinity
    arrays[1][:], arrays[3][:] = 127, 127
    arrays[2][0, 0, :40], arrays[2][0, 0, 40:] = 0x22, 0x44
    arrays[0][0, 0, 40:, 0] = 0x2A                        # channel 0 is -1: scores of +inf for -inf
    cache, _ = device_cache(arrays, d)
    out = strided(np.full(q.shape, 3.0, np.float32), dtype, "rows")
    _forward(strided(q, dtype, "rows"), cache, out)
    assert np.isnan(host(out)).all()                      # every row has a +inf
    arrays[0][0, 0, 40:, 0] = 0x22
    arrays[0][0, 0, :40, 0] = 0x22
    cache, _ = device_cache(arrays, d)
    _forward(strided(q, dtype, "rows"), cache, out)
    got = host(out)
    assert np.isnan(got[0, 1]).all() and (np.delete(got[0], 1, axis=0) == 0).all()  # all scores +inf; all -inf


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_no_slots_give_zeros_and_no_queries_only_carry(dtype):
    q = torch.randn(2, 5, 4, 64, device="cuda").to(dtype)
    none = si.Cache4.empty(2, 2, 0, 64)
    out = torch.full_like(q, 7.0)
    _forward(q, none, out, weight_out=torch.empty(2, 2, 0, device="cuda"))
    assert (out == 0).all()
    cache, _ = device_cache(random_cache(np.random.default_rng(0), 2, 2, 50, 64), 64)
    w, w_out = torch.rand(2, 2, 50, device="cuda"), torch.full((2, 2, 50), 5.0, device="cuda")
    _forward(q[:, :0], cache, out[:, :0], weight_in=w, weight_out=w_out, decay=0.5, k_len=lengths([50, 7]))
    assert torch.equal(w_out[0], w[0] * 0.5) and torch.equal(w_out[1, :, :7], w[1, :, :7] * 0.5) and (w_out[1, :, 7:] == 5).all()


def test_weights_in_place():
    rng = np.random.default_rng(5)
    cache, _ = device_cache(random_cache(rng, 1, 2, 300, 64), 64)
    q = torch.randn(1, 9, 4, 64, device="cuda", dtype=torch.bfloat16)
    w = torch.rand(1, 2, 300, device="cuda")
    apart, out = torch.empty_like(w), torch.empty_like(q)
    _forward(q, cache, out, weight_in=w, weight_out=apart, decay=0.9)
    _forward(q, cache, out, weight_in=w, weight_out=w, decay=0.9)
    assert torch.equal(w, apart)


@pytest.mark.parametrize("N", [1, 200])
def test_same_bits_every_time_on_any_stream_and_in_a_graph(N):
    rng = np.random.default_rng(6)
    cache, _ = device_cache(random_cache(rng, 2, 2, 9000, 64), 64)
    q = torch.randn(2, N, 8, 64, device="cuda", dtype=torch.bfloat16)
    ws = torch.empty(si.si_cache4_attn_workspace_bytes(q, cache, True), dtype=torch.uint8, device="cuda")
    k_len = lengths([9000, 777])
    ref, out = torch.empty_like(q), torch.empty_like(q)
    w_ref, w = torch.zeros(2, 2, 9000, device="cuda"), torch.zeros(2, 2, 9000, device="cuda")
    si.si_cache4_attn_forward(q, cache, ref, ws, k_len=k_len, weight_out=w_ref)
    torch.cuda.synchronize()
    for s in (None, torch.cuda.Stream()):
        out.zero_(), w.zero_()
        torch.cuda.synchronize()
        si.si_cache4_attn_forward(q, cache, out, ws, k_len=k_len, weight_out=w, stream=s)
        torch.cuda.synchronize()
        assert torch.equal(out, ref) and torch.equal(w, w_ref)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        si.si_cache4_attn_forward(q, cache, out, ws, k_len=k_len, weight_out=w)
    for i in range(3):
        q.normal_()
        k_len.copy_(torch.tensor([9000 - 1000 * i, 700 + i], dtype=torch.int32))
        w.zero_(), w_ref.zero_()
        si.si_cache4_attn_forward(q, cache, ref, ws, k_len=k_len, weight_out=w_ref)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, ref) and torch.equal(w, w_ref), i


def test_two_streams_with_workspaces_of_their_own():
    rng = np.random.default_rng(7)
    cache, _ = device_cache(random_cache(rng, 1, 2, 20000, 64), 64)
    qs = [torch.randn(1, 1, 8, 64, device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    refs, outs = [torch.empty_like(q) for q in qs], [torch.empty_like(q) for q in qs]
    for q, ref in zip(qs, refs):
        _forward(q, cache, ref)
    ws = [torch.empty(si.si_cache4_attn_workspace_bytes(qs[0], cache), dtype=torch.uint8, device="cuda") for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(10):
        for i in range(2):
            si.si_cache4_attn_forward(qs[i], cache, outs[i], ws[i], stream=streams[i])
    torch.cuda.synchronize()
    assert all(torch.equal(o, r) for o, r in zip(outs, refs))


def test_offsets_beyond_32_bits():
    """A cache whose codes pass 4 GiB: zeros (score 0, value 0), but for the last 100 slots of its last head."""
    cap, d = 36_000_000, 128
    cache = si.Cache4(*(torch.zeros(1, 2, cap, n, dtype=torch.uint8, device="cuda") for n in (64, 4, 64, 4)), d)
    arrays = random_cache(np.random.default_rng(8), 1, 1, 100, d)
    for t, a in zip(cache.tensors, arrays):
        t[:, 1:, -100:].copy_(torch.from_numpy(a).to("cuda"))
    for t in (cache.k_scales, cache.v_scales):
        t[:, :, :-100] = 127
        t[:, 0] = 127
    k, v = values(arrays, d)
    # queries along the keys' mean: scores of the last slots up to some tens, against 36 million zeros
    q = draw(np.random.default_rng(9), (1, 2, 2, d), "bf16", 3.0)
    q[0, :, 1] = torch.from_numpy(8 * k[0, 0, :2]).to(torch.bfloat16).double().numpy()
    out = torch.empty(1, 2, 2, d, device="cuda", dtype=torch.bfloat16)
    w = torch.zeros(1, 2, cap, device="cuda")
    _forward(strided(q, "bf16", "rows"), cache, out, weight_out=w)
    assert (out[:, :, 0] == 0).all()
    s = q[0, :, 1] @ k[0, 0].T / math.sqrt(d)
    top = np.maximum(s.max(axis=-1, keepdims=True), 0)
    p, rest = np.exp(s - top), (cap - 100) * np.exp(-top)
    total = p.sum(axis=-1, keepdims=True) + rest
    p /= total
    ref = p @ v[0, 0]
    spread = np.stack([p[i] @ np.abs(v[0, 0] - ref[i]) + (1 - p[i].sum()) * np.abs(ref[i]) for i in range(2)])
    # sums over the slots: a lane adds one term in 32 x 4 x 64 of them
    tol = output_bound(q[:, :, 1:], k, spread, p @ np.abs(v[0, 0]), ref, "bf16", 1 / math.sqrt(d), cap // 8192)
    assert (np.abs(host(out)[0, :, 1] - ref) <= tol).all()
    want = p.sum(axis=0)
    tol = weight_bound(q[:, :, 1:], k, want, 0 * want, "bf16", 1 / math.sqrt(d), cap // 8192, 2)
    assert (np.abs(host(w)[0, 1, -100:] - want) <= tol).all()
    assert bool((w[0, 0] > 0).all())
