"""Refusals of the operators of the cache in 4 bits: every one is an error code, before any GPU call, on a machine without a GPU.  And
the oracle's own pins."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import oracle
import paper_2411_01171_amd as si
from paper_2411_01171_amd import binding as B

NULL, SHAPE, DTYPE, ALIGN, WORKSPACE, ARG = 1, 2, 3, 5, 6, 7
FAR = 1 << 32
BASE, CACHE, WS, LEN, WEIGHT = FAR, 64 * FAR, 256 * FAR, 300 * FAR, 310 * FAR
by = C.byref


def heads(at=0, dtype=B.SI_BF16, Bn=2, N=30, H=4, d=64, strides=None, ptr=None):
    sb, sn, sh = strides or (N * H * d, H * d, d)
    return B._Heads(BASE + at if ptr is None else ptr, dtype, Bn, N, H, d, sb, sn, sh)


def cache(at=0, Bn=2, H=4, cap=500, d=64, **parts):
    p = {n: CACHE + at + i * FAR for i, n in enumerate(("k_codes", "k_scales", "v_codes", "v_scales"))}
    p.update(parts)
    return B._Cache4(*p.values(), Bn, H, cap, d)


def store(k=None, v=None, first=None, length=None, c=None, weight=None):
    return si.lib().si_cache4_store(by(k or heads()), by(v or heads(FAR)), first, length, by(c or cache()), weight, None)


def load(k=None, v=None, first=None, length=None, c=None):
    return si.lib().si_cache4_load(by(c or cache()), first, length, by(k or heads()), by(v or heads(FAR)), None)


def attn(q=None, c=None, scale=0.125, run=0, q_len=None, k_len=None, w_in=None, decay=1.0, w_out=None, out=None, ws=WS, nbytes=1 << 40):
    return si.lib().si_cache4_attn_forward(by(q or heads()), by(c or cache()), scale, run, q_len, k_len, w_in, decay, w_out, by(out or heads(FAR)), ws, nbytes, None)


def evict(c=None, k_len=None, weight=WEIGHT, keep=100, first=0, last=0, out=None, w_out=WEIGHT + FAR, kept=WEIGHT + 2 * FAR, out_len=WEIGHT + 3 * FAR, ws=WS,
          nbytes=1 << 40):
    return si.lib().si_cache4_evict(by(c or cache()), k_len, weight, keep, first, last, by(out or cache(8 * FAR, cap=100)), w_out, kept, out_len, ws, nbytes, None)


BAD_CACHES = (dict(d=20), dict(d=136), dict(d=0), dict(H=0), dict(Bn=0), dict(cap=-1), dict(cap=1 << 31), dict(H=1 << 16), dict(Bn=1 << 25), dict(Bn=1 << 20, H=4, cap=1 << 20))


def test_null_pointers():
    L = si.lib()
    assert L.si_cache4_store(None, by(heads()), None, None, by(cache()), None, None) == NULL
    assert L.si_cache4_store(by(heads()), None, None, None, by(cache()), None, None) == NULL
    assert L.si_cache4_store(by(heads()), by(heads(FAR)), None, None, None, None, None) == NULL
    assert L.si_cache4_load(None, None, None, by(heads()), by(heads(FAR)), None) == NULL
    assert L.si_cache4_attn_forward(None, by(cache()), 1.0, 0, None, None, None, 1.0, None, by(heads()), WS, 1 << 40, None) == NULL
    assert L.si_cache4_attn_forward(by(heads()), None, 1.0, 0, None, None, None, 1.0, None, by(heads(FAR)), WS, 1 << 40, None) == NULL
    assert L.si_cache4_attn_forward(by(heads()), by(cache()), 1.0, 0, None, None, None, 1.0, None, None, WS, 1 << 40, None) == NULL
    assert L.si_cache4_evict(None, None, WEIGHT, 5, 0, 0, by(cache()), WEIGHT, WEIGHT, WEIGHT, WS, 1 << 40, None) == NULL
    assert L.si_cache4_evict(by(cache()), None, WEIGHT, 5, 0, 0, None, WEIGHT, WEIGHT, WEIGHT, WS, 1 << 40, None) == NULL
    for part in ("k_codes", "k_scales", "v_codes", "v_scales"):
        assert store(c=cache(**{part: None})) == NULL and attn(c=cache(**{part: None})) == NULL and load(c=cache(**{part: None})) == NULL
        assert evict(c=cache(**{part: None})) == NULL and evict(out=cache(8 * FAR, cap=100, **{part: None})) == NULL
        for call in (store, attn, load, evict):
            assert call(c=cache(**{part: CACHE + 8})) == ALIGN
    assert attn(ws=None) == NULL and evict(ws=None) == NULL and evict(weight=None) == NULL and evict(w_out=None) == NULL
    assert evict(kept=None) == NULL and evict(out_len=None) == NULL
    assert store(k=heads(ptr=0)) == NULL and load(v=heads(ptr=0)) == NULL


@pytest.mark.parametrize("bad", BAD_CACHES, ids=str)
def test_sizes_of_the_cache(bad):
    d, H, Bn = bad.get("d", 64), bad.get("H", 4), bad.get("Bn", 2)
    like = dict(d=d, H=H, Bn=Bn)
    assert store(k=heads(**like), v=heads(FAR, **like), c=cache(**bad)) == SHAPE
    assert load(k=heads(**like), v=heads(FAR, **like), c=cache(**bad)) == SHAPE
    assert attn(q=heads(**like), out=heads(FAR, **like), c=cache(**bad)) == SHAPE
    assert evict(c=cache(**bad)) == SHAPE
    assert si.lib().si_cache4_attn_workspace_bytes(by(heads(**like)), by(cache(**bad)), 0) == 0
    assert si.lib().si_cache4_evict_workspace_bytes(by(cache(**bad)), 10) == 0


def test_operands_that_do_not_fit_the_cache():
    for bad in (dict(H=3), dict(Bn=1), dict(d=32)):
        assert store(k=heads(**bad)) == SHAPE and store(v=heads(FAR, **bad)) == SHAPE, bad
        assert load(k=heads(**bad)) == SHAPE and load(v=heads(FAR, **bad)) == SHAPE, bad
    assert store(v=heads(FAR, N=29)) == SHAPE and store(v=heads(FAR, dtype=B.SI_F32)) == DTYPE and store(k=heads(dtype=7)) == DTYPE
    assert attn(q=heads(H=6)) == SHAPE and attn(q=heads(Bn=1)) == SHAPE and attn(q=heads(d=32)) == SHAPE
    assert attn(out=heads(FAR, H=8)) == SHAPE and attn(out=heads(FAR, N=31)) == SHAPE and attn(out=heads(FAR, dtype=B.SI_F32)) == DTYPE
    assert attn(run=-1) == SHAPE and attn(run=1 << 31) == SHAPE
    assert evict(out=cache(8 * FAR, cap=99)) == SHAPE and evict(out=cache(8 * FAR, cap=100, H=3)) == SHAPE and evict(out=cache(8 * FAR, cap=100, d=32)) == SHAPE
    assert evict(out=cache(8 * FAR, cap=100, Bn=1)) == SHAPE
    assert evict(keep=0) == SHAPE and evict(keep=-4) == SHAPE and evict(keep=1 << 31) == SHAPE
    # rows of a key head past 31 bits
    many = dict(Bn=1, N=1 << 30, H=4, d=8, strides=(1 << 36, 32, 8))
    assert attn(q=heads(**many), out=heads(1 << 40, **many), c=cache(Bn=1, H=1, d=8)) == SHAPE
    # more groups of tokens than 32 bits count
    long = dict(Bn=1 << 14, N=1 << 25, H=4, d=8, strides=(1 << 30, 32, 8))    # 2^33 of 256 tokens each
    assert store(k=heads(**long), v=heads(1 << 47, **long), c=cache(Bn=1 << 14, d=8)) == SHAPE


def test_arguments():
    for bad in (0.0, -1.0, math.nan, math.inf):
        assert attn(scale=bad) == ARG, bad
    assert attn(w_in=WEIGHT) == ARG                                              # carried over to nowhere
    for bad in (-1.0, math.nan, math.inf):
        assert attn(w_in=WEIGHT, w_out=WEIGHT, decay=bad) == ARG, bad
    for first, last in ((-1, 0), (0, -1), (101, 0), (0, 101), (60, 41), (1 << 62, 1 << 62)):
        assert evict(first=first, last=last) == ARG, (first, last)
    assert attn(ws=WS + 64) == ALIGN and evict(ws=WS + 64) == ALIGN
    for p in (LEN + 1, LEN + 2):
        assert store(first=p) == ALIGN and store(length=p) == ALIGN and store(weight=p) == ALIGN and load(first=p) == ALIGN
        assert attn(q_len=p) == ALIGN and attn(k_len=p) == ALIGN and attn(w_out=p) == ALIGN and attn(w_in=p, w_out=WEIGHT) == ALIGN
        assert evict(k_len=p) == ALIGN and evict(weight=p) == ALIGN and evict(w_out=p) == ALIGN and evict(kept=p) == ALIGN and evict(out_len=p) == ALIGN


def test_workspaces():
    L = si.lib()
    one, long = heads(N=1, H=32, Bn=1, d=128), cache(cap=100000, H=8, Bn=1, d=128)
    plain, weights = (L.si_cache4_attn_workspace_bytes(by(one), by(long), w) for w in (0, 1))
    assert weights > plain > 1 << 16                                             # the shares of a token that is dealt out
    out = heads(FAR, N=1, H=32, Bn=1, d=128)
    assert attn(q=one, c=long, out=out, nbytes=plain - 1) == WORKSPACE
    assert attn(q=one, c=long, out=out, w_out=WEIGHT, nbytes=plain) == WORKSPACE
    n = L.si_cache4_evict_workspace_bytes(by(cache()), 100)
    assert n > 0 and evict(nbytes=n - 1) == WORKSPACE
    assert L.si_cache4_evict_workspace_bytes(by(cache()), 0) == 0


def test_operands_that_overlap():
    c = cache()
    for at in (c.k_codes, c.k_scales, c.v_codes, c.v_scales):
        inside = at + 4096 if at in (c.k_codes, c.v_codes) else at + 1024
        assert store(k=heads(ptr=inside)) == ARG and store(v=heads(ptr=inside)) == ARG and store(weight=inside) == ARG and store(first=inside) == ARG
        assert load(k=heads(ptr=inside)) == ARG and load(v=heads(ptr=inside)) == ARG
        assert attn(out=heads(ptr=inside)) == ARG and attn(ws=inside) == ARG and attn(w_out=inside) == ARG
        assert evict(w_out=inside) == ARG and evict(kept=inside) == ARG and evict(out_len=inside) == ARG and evict(ws=inside) == ARG
    assert store(c=cache(k_scales=CACHE + 64)) == ARG and store(c=cache(v_codes=CACHE)) == ARG      # arrays of one cache
    assert load(c=cache(v_codes=CACHE), v=heads()) == ARG                        # (reading, they may be one:) two outputs in one place
    assert load(k=heads(), v=heads(64 * 2)) == ARG and load(k=heads(strides=(7680, 0, 64))) == ARG
    assert load(first=BASE) == ARG and load(length=BASE + FAR + 8) == ARG
    assert store(weight=BASE + 64) == ARG and store(weight=WEIGHT, first=WEIGHT + 4) == ARG and store(weight=WEIGHT, length=WEIGHT) == ARG
    assert attn(out=heads()) == ARG and attn(out=heads(64)) == ARG and attn(out=heads(FAR, strides=(7680, 0, 64))) == ARG
    assert attn(ws=BASE) == ARG and attn(ws=BASE + FAR) == ARG and attn(w_out=BASE + 64) == ARG and attn(w_out=BASE + FAR) == ARG
    assert attn(w_out=WS) == ARG and attn(w_in=WS, w_out=WEIGHT) == ARG and attn(w_in=WEIGHT + 4, w_out=WEIGHT) == ARG and attn(w_in=BASE + FAR, w_out=WEIGHT) == ARG
    assert attn(q_len=WS) == ARG and attn(k_len=WS + 4) == ARG and attn(k_len=BASE + FAR) == ARG and attn(k_len=WEIGHT, w_out=WEIGHT) == ARG
    # the target of an eviction: its source, a part of it, its own weights
    assert evict(out=cache()) == ARG and evict(out=cache(4096, cap=100)) == ARG and evict(out=cache(8 * FAR, cap=100, k_scales=CACHE + 8 * FAR + 64)) == ARG
    assert evict(w_out=WEIGHT) == ARG and evict(kept=WEIGHT + 64) == ARG and evict(out_len=WEIGHT) == ARG and evict(kept=WEIGHT + FAR) == ARG
    assert evict(k_len=WEIGHT + FAR) == ARG and evict(k_len=WEIGHT + 3 * FAR) == ARG and evict(out_len=WEIGHT + 2 * FAR) == ARG
    assert evict(ws=WEIGHT) == ARG and evict(ws=WEIGHT + FAR) == ARG and evict(ws=WEIGHT + 3 * FAR) == ARG


def test_binding_refuses_what_it_cannot_describe():
    new = lambda *n: torch.zeros(1, 2, 50, *n, dtype=torch.uint8)  # noqa: E731
    good = si.Cache4(new(32), new(2), new(32), new(2), 64)
    assert good.shape == (1, 2, 50, 64) and si.Cache4.empty(1, 2, 50, 72, device="cpu").k_codes.shape[3] == 48
    for bad in ((new(16), new(2), new(32), new(2), 64), (new(32), new(1), new(32), new(2), 64), (new(32).int(), new(2), new(32), new(2), 64),
                (new(32), new(2), new(32)[:, :, ::2], new(2), 64), (new(32), new(2), new(64)[..., ::2], new(2), 64), (new(32), new(2), new(32), new(2), 20),
                (new(32), new(2), new(32), new(2), 136)):
        with pytest.raises(ValueError):
            si.Cache4(*bad)
    x, w, ws = torch.zeros(1, 4, 2, 64), torch.zeros(1, 2, 50), torch.zeros(1 << 16, dtype=torch.uint8)
    calls = (lambda: si.si_cache4_store(x, x, good),                                              # not on a GPU
             lambda: si.si_cache4_store(x, x, good, first=torch.zeros(1)), lambda: si.si_cache4_store(x, x, good, length=torch.zeros(2, dtype=torch.int32)),
             lambda: si.si_cache4_store(x, x, good, weight=w.double()), lambda: si.si_cache4_store(x, x, good, weight=w[:, :, 1:]),
             lambda: si.si_cache4_load(good, x[0], x), lambda: si.si_cache4_attn_forward(x, good, x.clone(), ws, weight_out=w[0]),
             lambda: si.si_cache4_attn_forward(x, good, x.clone(), ws, weight_in=w.t() if w.dim() == 2 else w.transpose(1, 2), weight_out=w),
             lambda: si.si_cache4_evict(good, w, 10, good, w, torch.zeros(1, 2, 11, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), ws),
             lambda: si.si_cache4_evict(good, w, 10, good, w, torch.zeros(1, 2, 10), torch.zeros(1, dtype=torch.int32), ws),
             lambda: si.si_cache4_evict(good, w, 10, good, w, torch.zeros(1, 2, 10, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), ws))
    for i, call in enumerate(calls):
        with pytest.raises(ValueError):
            call()


# ------------------------------------------------------------------------------------------------ the oracle's pins

def test_groups_by_hand():
    codes, s = oracle.encode_group_ref([6.0, -6.0, 3.0, 0.25, 0.75, -5.0, 2.5, 1.0])
    assert s == 127 and codes.tolist() == [7, 15, 5, 0, 2, 14, 4, 2]             # 0.25, 0.75, 5, 2.5: ties to the even code
    codes, s = oracle.encode_group_ref([7.0, 6.9])
    assert s == 127 and codes.tolist() == [7, 7]
    codes, s = oracle.encode_group_ref([7.001, 6.0])
    assert s == 128 and codes.tolist() == [6, 5]  # 3.5005 is nearer to 4, 3 is itself
    assert oracle.encode_group_ref([0.0, -0.0])[0].tolist() == [0, 8] and oracle.encode_group_ref([0.0])[1] == 2
    assert oracle.encode_group_ref([1.0, math.nan]) [1] == 255 and oracle.encode_group_ref([math.inf])[1] == 255
    assert oracle.encode_group_ref([3.4e38])[1] == 252
    assert [oracle.scale_room_ref(d) for d in (8, 32, 40, 72, 96, 104, 128)] == [(1, 1), (1, 1), (2, 2), (3, 4), (3, 4), (4, 4), (4, 4)]


def test_codes_survive_a_round_trip():
    """What a code stands for is stored as that code again, if its group's largest is more than 3.5 units."""
    rng = np.random.default_rng(0)
    codes, scales = rng.integers(0, 256, (20, 32), dtype=np.uint8), rng.integers(2, 253, (20, 2), dtype=np.uint8)
    codes[:, [0, 16]] = 0x76  # a 4 and a 6 in every group
    held = oracle.decode_ref(codes, scales, 64)
    again = oracle.encode_ref(held)
    assert (again[0] == codes).all() and (again[1] == scales).all()
    x = rng.standard_normal((50, 40))
    held = oracle.decode_ref(*oracle.encode_ref(x), 40)
    assert np.abs(held - x).max() <= np.abs(x).max() / 6 and np.corrcoef(held.ravel(), x.ravel())[0, 1] > 0.99


def test_attention_against_the_reference_of_heads():
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal((2, 7, 4, 16)), rng.standard_normal((2, 2, 50, 16)), rng.standard_normal((2, 2, 50, 16))
    back = lambda t: t.transpose(0, 2, 1, 3)  # noqa: E731
    for k_len in (None, [50, 9]):
        a = oracle.cache_attention_ref(q, k, v, k_len=k_len)
        b = oracle.sparse_attention_ref(q, back(k), back(v), None, 7, 64, k_len=k_len)
        for x, y in zip(a[:3], b):
            assert np.allclose(x, y, atol=1e-12)
        # every row hands out a weight of one
        assert np.allclose(np.nansum(a[3], axis=-1), 7 * 2)
    # runs: every run on its own, over what lies before its end
    whole = oracle.cache_attention_ref(q, k, v, run=3)[0]
    for n in range(7):
        end = 50 - 7 + min((n // 3 + 1) * 3, 7)
        assert np.allclose(whole[:, n:n + 1], oracle.cache_attention_ref(q[:, n:n + 1], k[:, :, :end], v[:, :, :end])[0], atol=1e-12)
    assert oracle.seen_ref(0, 5, 3, 1) == 0 and oracle.seen_ref(2, 5, 3, 1) == 1 and oracle.seen_ref(4, 5, 3, 1) == 3


def test_eviction_by_hand():
    w = np.array([[[5.0, 1.0, np.nan, 3.0, 3.0, -np.inf, 0.0, 9.0]]])
    assert oracle.evict_ref(w, 3) == [[[0, 3, 7]]] and oracle.evict_ref(w, 4) == [[[0, 3, 4, 7]]] and oracle.evict_ref(w, 6) == [[[0, 1, 3, 4, 6, 7]]]
    assert oracle.evict_ref(w, 7) == [[[0, 1, 2, 3, 4, 6, 7]]]                   # NaN ties with -infinity: the lower slot
    assert oracle.evict_ref(w, 3, first=2, last=1) == [[[0, 1, 7]]] and oracle.evict_ref(w, 4, first=1, last=1) == [[[0, 3, 4, 7]]]
    assert oracle.evict_ref(w, 3, k_len=[5]) == [[[0, 3, 4]]] and oracle.evict_ref(w, 8) == [[list(range(8))]] and oracle.evict_ref(w, 3, k_len=[2]) == [[[0, 1]]]
