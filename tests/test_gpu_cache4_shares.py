"""Attention over the cache in 4 bits where a tile's keys are dealt out to several workgroups, and workgroups that take a second tile."""
import math

import numpy as np
import pytest
import torch

import oracle
import paper_2411_01171_amd as si
from attn_helpers import draw, host, lengths, strided
from cache4_helpers import device_cache, output_bound, random_cache, values
from gpu_helpers import guarded, guards_intact
from test_gpu_cache4_attn import _check, _forward

pytestmark = pytest.mark.gpu


def _shared(dtype, B, N, cap, Hq, Hk, d):
    """Whether the outputs of two shares at least have room in the workspace."""
    q = torch.empty(B, N, Hq, d, dtype=torch.float32 if dtype == "f32" else torch.bfloat16)
    cache = si.Cache4.empty(B, Hk, cap, d, device="cpu")
    return si.si_cache4_attn_workspace_bytes(q, cache) >= 2 * B * N * Hq * d * 4


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 80, 128])
@pytest.mark.parametrize("run,group", [(129, 1), (160, 2), (200, 1), (399, 1), (256, 1)])
def test_tiles_that_end_with_their_run(dtype, d, run, group):
    """Tiles of 128 and 256 rows of one run each; early runs see fewer keys than the last, padded ones none."""
    B, N, cap = 3, 400, 5000
    assert _shared(dtype, B, N, cap, group, 1, d)
    _check(dtype, B, N, cap, group, 1, d, run=run, q_len=[400, 300, 131], k_len=[4800, 250, 5000])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,run", [(6, 0), (6, 1), (150, 0), (150, 50), (300, 150)])
@pytest.mark.parametrize("which", ["key", "value"])
@pytest.mark.parametrize("at", [1, 2500, 4990])
def test_not_finite_in_one_share(dtype, N, run, which, at):
    rng = np.random.default_rng(12)
    d, cap = 96, 5000
    assert _shared(dtype, 1, N, cap, 2, 2, d)
    q = draw(rng, (1, N, 2, d), dtype)
    arrays = [a.copy() for a in random_cache(rng, 1, 2, cap, d)]
    if at == 4990:
        at = cap - N // 2  # seen by the later runs only
    arrays[1 if which == "key" else 3][0, 1, at, 1] = 255
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
    ref2, spread, mass, _ = oracle.cache_attention_ref(q, k, v, run)
    ok = ~np.isnan(ref)
    tol = output_bound(q, k, spread, mass, ref2, dtype, 1 / math.sqrt(d), cap)
    assert (np.abs(host(out) - ref2)[ok] <= tol[ok]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [2, 150])
@pytest.mark.parametrize("at", [0, 2500, 4999])
def test_infinite_queries_in_one_share(dtype, N, at):
    """A score of +inf in one share makes a row NaN, and what it gives to every slot; scores of -inf weigh nothing, and rows that have no other give zeros."""
    d, cap = 32, 5000
    assert _shared(dtype, 1, N, cap, 1, 1, d)
    q = np.zeros((1, N, 1, d), np.float32)
    q[0, :, 0, 0] = -np.inf
    arrays = [np.full((1, 1, cap, n), fill, np.uint8) for n, fill in ((16, 0x22), (1, 127), (16, 0x22), (1, 127))]  # ones

    def run():
        cache, _ = device_cache(arrays, d)
        out, w = strided(np.full(q.shape, 3.0, np.float32), dtype, "rows"), torch.full((1, 1, cap), 5.0, device="cuda")
        _forward(strided(q, dtype, "rows"), cache, out, weight_out=w)
        return host(out), host(w)

    out, w = run()
    assert (out == 0).all() and (w == 0).all()
    arrays[0][0, 0, at, 0] = 0x2A  # channel 0 is -1
    out, w = run()
    assert np.isnan(out).all() and np.isnan(w).all()
    q[0, :, 0, 0] = np.inf  # now all slots but one have +inf
    out, w = run()
    assert np.isnan(out).all() and np.isnan(w).all()


@pytest.mark.parametrize("dtype,N", [(torch.bfloat16, 100), (torch.bfloat16, 130), (torch.float32, 100)])
def test_more_tiles_of_many_rows_than_workgroups(dtype, N):
    """Tiles of 128 and 256 rows, more of them than a launch has workgroups: some heads against calls of their own, and values that are not finite in
    every third head show there only."""
    gen = torch.Generator(device="cuda").manual_seed(2)
    b, h, cap = 1030, 1024, 40
    q = torch.randn(b, N, h, 8, generator=gen, device="cuda", dtype=dtype)
    cache = si.Cache4(*(torch.randint(0, 256, (b, h, cap, c), generator=gen, device="cuda", dtype=torch.uint8) if c == 16
                        else torch.full((b, h, cap, 1), 126, device="cuda", dtype=torch.uint8) for c in (16, 1, 16, 1)), 8)
    for t in (cache.k_codes, cache.v_codes):
        t[..., 4:] = 0
    bad = torch.arange(b * h, device="cuda").view(b, h) % 3 == 1
    cache.v_scales[:, :, 7, 0] = torch.where(bad, 255, 126).to(torch.uint8)
    out, weight = torch.empty_like(q), torch.empty(b, h, cap, device="cuda")
    n = si.si_cache4_attn_workspace_bytes(q, cache, True)
    buf, ws = guarded(n)
    si.si_cache4_attn_forward(q, cache, out, ws, weight_out=weight)
    assert guards_intact(buf, n)
    for at in range(0, b, 103):
        assert torch.equal(out[at].isnan(), bad[at].view(1, h, 1).expand(N, h, 8))
    assert bool(weight.isfinite().all())
    for at in (0, 1, h // 2, h - 2, h - 1):
        part = si.Cache4(*(t[:, at:at + 1].contiguous() for t in cache.tensors), 8)
        o, w = torch.empty(b, N, 1, 8, device="cuda", dtype=dtype), torch.empty(b, 1, cap, device="cuda")
        ws = torch.empty(si.si_cache4_attn_workspace_bytes(o, part, True), dtype=torch.uint8, device="cuda")
        si.si_cache4_attn_forward(q[:, :, at:at + 1].contiguous(), part, o, ws, weight_out=w)
        fine = ~bad[:, at]
        assert torch.equal(o[fine], out[fine][:, :, at:at + 1]) and torch.equal(w, weight[:, at:at + 1]), at


def test_rotated_keys_in_the_cache():
    """Frames of tokens whose positions are rotated, then stored, then seen by the rotated queries of the next frame."""
    rng = np.random.default_rng(14)
    B, Hq, Hk, d, h, w, frames = 2, 4, 2, 64, 5, 7, 3
    rope = si.Rope((frames, h, w), (8, 12, 12))
    frame = h * w
    cache, intact = device_cache(random_cache(rng, B, Hk, frames * frame, d), d)
    keys, vals = [], []
    for f in range(frames):
        q, k, v = draw(rng, (B, frame, Hq, d), "bf16"), draw(rng, (B, frame, Hk, d), "bf16"), draw(rng, (B, frame, Hk, d), "bf16")
        dq, dk, dv = (strided(t, "bf16", "projection") for t in (q, k, v))
        rq, rk = torch.empty(B, frame, Hq, d, device="cuda", dtype=dq.dtype), torch.empty(B, frame, Hk, d, device="cuda", dtype=dq.dtype)
        si.si_rope_forward(dq, dk, rope, rq, rk, first=f * frame)
        si.si_cache4_store(rk, dv, cache, first=lengths([f * frame] * B))
        out = torch.empty_like(rq)
        _forward(rq, cache, out, k_len=lengths([(f + 1) * frame] * B))
        if f:
            assert not torch.equal(rk, dk)
        keys.append(oracle.decode_ref(*oracle.encode_ref(host(rk)), d))
        vals.append(oracle.decode_ref(*oracle.encode_ref(v), d))
        kk, vv = (np.concatenate(x, axis=1).transpose(0, 2, 1, 3) for x in (keys, vals))
        ref, spread, mass, _ = oracle.cache_attention_ref(host(rq), kk, vv)
        assert (np.abs(host(out) - ref) <= output_bound(host(rq), kk, spread, mass, ref, "bf16", 1 / math.sqrt(d), kk.shape[2])).all(), f
    assert intact()
