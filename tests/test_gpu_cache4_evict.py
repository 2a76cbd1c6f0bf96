"""si_cache4_evict against the oracle, exactly, and the operators of the cache one after the other."""
import math

import numpy as np
import pytest
import torch

import oracle
import paper_2411_01171_amd as si
from attn_helpers import draw, host, lengths, strided
from cache4_helpers import device_cache, output_bound, random_cache, values, weight_bound
from gpu_helpers import guarded, guards_intact

pytestmark = pytest.mark.gpu


def _evict(cache, w, keep, out, w_out, kept, out_len, **kw):
    n = si.si_cache4_evict_workspace_bytes(cache, keep)
    assert n > 0
    buf, ws = guarded(n)
    si.si_cache4_evict(cache, w, keep, out, w_out, kept, out_len, ws, **kw)
    torch.cuda.synchronize()
    assert guards_intact(buf, n)


def _check(B, heads, cap, d, keep, first=0, last=0, k_len=None, weight=None, out_cap=None, seed=0):
    rng = np.random.default_rng(seed)
    arrays = random_cache(rng, B, heads, cap, d)
    w = rng.random((B, heads, cap)).astype(np.float32) if weight is None else np.ascontiguousarray(weight, np.float32)
    room = max(1, min(keep, cap)) if out_cap is None else out_cap
    target = random_cache(rng, B, heads, room, d)
    cache, intact = device_cache(arrays, d)
    out, out_intact = device_cache(target, d)
    w_buf, w_out = guarded(torch.empty(B, heads, room, device="cuda"))
    w_out.fill_(5.0)
    k_buf, kept = guarded(torch.empty(B, heads, keep, dtype=torch.int32, device="cuda"))
    kept.fill_(-9)
    out_len = torch.full((B,), -9, dtype=torch.int32, device="cuda")
    _evict(cache, torch.from_numpy(w).to("cuda"), keep, out, w_out, kept, out_len, first=first, last=last, k_len=lengths(k_len))
    assert intact() and out_intact() and guards_intact(w_buf, w_out.nbytes) and guards_intact(k_buf, kept.nbytes)
    stay = oracle.evict_ref(w, keep, first, last, k_len)
    want = [a.copy() for a in target]
    w_want, kept_want = np.full((B, heads, room), 5.0, np.float32), np.full((B, heads, keep), -9, np.int32)
    for b in range(B):
        for h in range(heads):
            m = len(stay[b][h])
            for a, from_ in zip(want, arrays):
                a[b, h, :m] = from_[b, h, stay[b][h]]
            w_want[b, h, :m], kept_want[b, h, :m] = w[b, h, stay[b][h]], stay[b][h]
        assert int(out_len[b]) == len(stay[b][0])
    assert np.array_equal(kept.cpu().numpy(), kept_want)
    assert np.array_equal(w_out.cpu().numpy(), w_want, equal_nan=True)
    for t, a in zip(out.tensors, want):
        assert np.array_equal(t.cpu().numpy(), a)


@pytest.mark.parametrize("d", range(8, 129, 8))
def test_head_widths(d):
    _check(2, 3, 200, d, 70, first=2, last=9)


@pytest.mark.parametrize("cap", [1, 2, 63, 64, 65, 1000, 1023, 1024, 1025, 2048, 4097, 16384, 16385, 32768, 32769, 33000, 70001])
@pytest.mark.parametrize("share", [0.0, 0.3, 0.99, 1.0, 1.5])
def test_lengths(cap, share):
    _check(1, 2, cap, 32, max(1, int(cap * share)), seed=cap)


@pytest.mark.parametrize("k_len", [[0, 100, 5000], [-1, 99, 101], [9999, 1, 4999]])
@pytest.mark.parametrize("first,last", [(0, 0), (100, 0), (0, 100), (30, 70), (4, 20)])
def test_padded_batches_and_protected_slots(k_len, first, last):
    _check(3, 2, 5000, 64, 100, first=first, last=last, k_len=k_len)


@pytest.mark.parametrize("cap", [300, 20000, 60000])
@pytest.mark.parametrize("kind", ["equal", "two", "zeros", "steps", "neighbours", "wide", "special"])
def test_weights_with_ties_and_of_every_kind(cap, kind):
    rng = np.random.default_rng(1)
    shape = (1, 3, cap)
    w = {"equal": lambda: np.full(shape, 0.125), "two": lambda: (rng.random(shape) < 0.3).astype(np.float32),
         "zeros": lambda: np.where(rng.random(shape) < 0.7, 0.0, rng.random(shape)),
         "steps": lambda: rng.integers(0, 50, shape) / 16.0,
         "neighbours": lambda: np.float32(1.0) + rng.integers(0, 8, shape) * np.float32(2.0 ** -23),
         "wide": lambda: np.exp(rng.standard_normal(shape) * 20),
         "special": lambda: rng.choice(np.array([np.nan, np.inf, -np.inf, 0.0, -0.0, 1e-45, -1e-45, 1.0, -1.0, 3e38, -3e38], np.float32), shape)}[kind]()
    for keep in (1, cap // 3, cap - 1):
        _check(1, 3, cap, 16, keep, weight=w)
        _check(1, 3, cap, 16, keep, first=min(1, keep - 1), last=(keep - 1) // 2, weight=w)


def test_many_lists_and_a_larger_target():
    _check(5, 70, 90, 40, 30, last=7, k_len=[90, 31, 30, 29, 0], out_cap=33)


def test_empty_cache():
    cache, out = si.Cache4.empty(2, 3, 0, 64), si.Cache4.empty(2, 3, 5, 64)
    out_len = torch.full((2,), -9, dtype=torch.int32, device="cuda")
    _evict(cache, torch.empty(2, 3, 0, device="cuda"), 5, out, torch.zeros(2, 3, 5, device="cuda"), torch.zeros(2, 3, 5, dtype=torch.int32, device="cuda"), out_len)
    assert (out_len == 0).all()


@pytest.mark.parametrize("cap", [3000, 50000])
def test_in_a_graph_and_on_another_stream(cap):
    rng = np.random.default_rng(2)
    cache, _ = device_cache(random_cache(rng, 2, 2, cap, 64), 64)
    keep = cap // 4
    w = torch.rand(2, 2, cap, device="cuda")
    k_len = lengths([cap, cap // 2])
    ws = torch.empty(si.si_cache4_evict_workspace_bytes(cache, keep), dtype=torch.uint8, device="cuda")
    new = lambda: (si.Cache4(*(torch.zeros(2, 2, keep, n, dtype=torch.uint8, device="cuda") for n in (32, 2, 32, 2)), 64), torch.zeros(2, 2, keep, device="cuda"),  # noqa: E731
                   torch.zeros(2, 2, keep, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda"))
    ref, got = new(), new()
    same = lambda: all(torch.equal(a, b) for a, b in zip((*ref[0].tensors, *ref[1:]), (*got[0].tensors, *got[1:])))  # noqa: E731
    si.si_cache4_evict(cache, w, keep, *ref, ws, first=2, last=10, k_len=k_len)
    torch.cuda.synchronize()
    si.si_cache4_evict(cache, w, keep, *got, ws, first=2, last=10, k_len=k_len, stream=torch.cuda.Stream())
    torch.cuda.synchronize()
    assert same()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        si.si_cache4_evict(cache, w, keep, *got, ws, first=2, last=10, k_len=k_len)
    for i in range(3):
        w.uniform_()
        k_len.copy_(torch.tensor([cap - i, cap // (i + 2)], dtype=torch.int32))
        for t in (*ref[0].tensors, *ref[1:], *got[0].tensors, *got[1:]):
            t.zero_()
        si.si_cache4_evict(cache, w, keep, *ref, ws, first=2, last=10, k_len=k_len)
        graph.replay()
        torch.cuda.synchronize()
        assert same(), i


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_stream_of_frames(dtype):
    """Frames come one by one: stored, attended with their predecessors, and once the cache is full the slots with the least weight leave."""
    rng = np.random.default_rng(3)
    B, Hq, Hk, d, frame, cap, keep = 2, 4, 2, 40, 30, 128, 70
    caches = [si.Cache4(*(torch.full((B, Hk, cap, n), 0xFF, dtype=torch.uint8, device="cuda") for n in (32, 2, 32, 2)), d) for _ in range(2)]
    weights = [torch.full((B, Hk, cap), math.nan, device="cuda") for _ in range(2)]
    n_dev = torch.zeros(B, dtype=torch.int32, device="cuda")
    ws_attn = ws_evict = None
    model = [[([], [], []) for _ in range(Hk)] for _ in range(B)]  # keys, values, weights of what the cache should hold
    now = 0
    for step in range(9):
        q, k, v = draw(rng, (B, frame, Hq, d), dtype), draw(rng, (B, frame, Hk, d), dtype), draw(rng, (B, frame, Hk, d), dtype)
        kq, vq = (oracle.decode_ref(*oracle.encode_ref(t), d) for t in (k, v))
        dq, dk, dv = (strided(t, dtype, "projection") for t in (q, k, v))
        cache, weight = caches[now], weights[now]
        si.si_cache4_store(dk, dv, cache, first=n_dev, weight=weight)
        n_dev.add_(frame)
        out = torch.empty(B, frame, Hq, d, device="cuda", dtype=dq.dtype)
        if ws_attn is None:
            ws_attn = torch.empty(si.si_cache4_attn_workspace_bytes(dq, cache, True), dtype=torch.uint8, device="cuda")
            ws_evict = torch.empty(si.si_cache4_evict_workspace_bytes(cache, keep), dtype=torch.uint8, device="cuda")
        si.si_cache4_attn_forward(dq, cache, out, ws_attn, k_len=n_dev, weight_in=weight, weight_out=weight, decay=0.5)
        for b in range(B):
            for h in range(Hk):
                ks, vs, w = model[b][h]
                ks.extend(kq[b, :, h]), vs.extend(vq[b, :, h]), w.extend([0.0] * frame)
        n = len(model[0][0][0])
        keys, vals, old = (np.array([[model[b][h][x] for h in range(Hk)] for b in range(B)]) for x in range(3))
        ref, spread, mass, w_ref = oracle.cache_attention_ref(q, keys, vals, 0, None, None, None, old, 0.5)
        assert (np.abs(host(out) - ref) <= output_bound(q, keys, spread, mass, ref, dtype, 1 / math.sqrt(d), n)).all(), step
        w_got = host(weight[:, :, :n])
        tol = weight_bound(q, keys, w_ref - 0.5 * old, 0.5 * old, dtype, 1 / math.sqrt(d), n, 2 * frame)
        assert (np.abs(w_got - w_ref) <= tol).all(), step
        for b in range(B):  # the model goes on with the weights that the library has, so that both choose by the same ones
            for h in range(Hk):
                model[b][h][2][:] = list(w_got[b, h])
        if n + frame > cap:
            kept, out_len = torch.full((B, Hk, keep), -1, dtype=torch.int32, device="cuda"), torch.empty(B, dtype=torch.int32, device="cuda")
            si.si_cache4_evict(cache, weight, keep, caches[1 - now], weights[1 - now], kept, out_len, ws_evict, first=2, last=frame, k_len=n_dev)
            stay = oracle.evict_ref(w_got, keep, 2, frame)
            assert np.array_equal(kept.cpu().numpy(), np.array(stay))
            for b in range(B):
                for h in range(Hk):
                    model[b][h] = tuple([part[i] for i in stay[b][h]] for part in model[b][h])
            n_dev.copy_(out_len)
            now = 1 - now
