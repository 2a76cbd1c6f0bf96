"""Refusals of the operators on heads of video tokens and of the block that uses them: every one is an error code, before any
GPU call, on a machine without a GPU.  And the oracle's own pins."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import oracle
import paper_2411_01171_amd as si
import si_workloads as wl
from paper_2411_01171_amd import binding as B

NULL, SHAPE, DTYPE, SLICE, ALIGN, WORKSPACE, ARG = 1, 2, 3, 4, 5, 6, 7
BASE, WS, BITS, LEN = 0x100000000, 0x700000000000, 0x7100000000, 0x7200000000


def heads(at=0, dtype=B.SI_BF16, Bn=2, N=300, H=4, d=64, strides=None, ptr=None):
    sb, sn, sh = strides or (N * H * d, H * d, d)
    return B._Heads(BASE + at if ptr is None else ptr, dtype, Bn, N, H, d, sb, sn, sh)


FAR = 1 << 32  # an operand of its own


def rope(pairs=(8, 12, 12), extent=(3, 10, 10), **kw):
    s = si.Rope(extent, pairs).struct
    for k, v in kw.items():
        if k in ("origin", "step"):
            getattr(s, k)[:] = list(v)
        else:
            setattr(s, k, v)
    return s


def rope_call(q=None, k=None, r=None, first=0, qo=None, ko=None, lone=False):
    q = q or heads()
    k = None if lone else k or heads(FAR)
    qo, ko = qo or heads(2 * FAR), (None if lone else ko or heads(3 * FAR))
    by = lambda t: None if t is None else C.byref(t)  # noqa: E731
    return si.lib().si_rope_forward(by(q), by(k), C.byref(r or rope()), first, by(qo), by(ko), None)


def test_rope_refusals():
    assert si.lib().si_rope_forward(None, None, C.byref(rope()), 0, None, None, None) == NULL
    assert si.lib().si_rope_forward(C.byref(heads()), C.byref(heads(FAR)), None, 0, C.byref(heads(2 * FAR)), C.byref(heads(3 * FAR)), None) == NULL
    assert si.lib().si_rope_forward(C.byref(heads()), C.byref(heads(FAR)), C.byref(rope()), 0, C.byref(heads(2 * FAR)), None, None) == NULL
    assert rope_call(q=heads(ptr=0)) == NULL and rope_call(qo=heads(ptr=0)) == NULL
    assert rope_call(q=heads(dtype=5)) == DTYPE and rope_call(k=heads(FAR, dtype=B.SI_F32)) == DTYPE and rope_call(qo=heads(2 * FAR, dtype=B.SI_F32)) == DTYPE
    for bad in (dict(d=20), dict(d=136), dict(d=0), dict(H=0), dict(Bn=0), dict(N=-1), dict(N=1 << 31)):
        assert rope_call(q=heads(**bad)) == SHAPE, bad
    assert rope_call(k=heads(FAR, N=299)) == SHAPE and rope_call(k=heads(FAR, Bn=1)) == SHAPE and rope_call(k=heads(FAR, d=32)) == SHAPE
    assert rope_call(qo=heads(2 * FAR, H=5)) == SHAPE
    assert rope_call(q=heads(ptr=BASE + 8)) == ALIGN and rope_call(q=heads(strides=(76800, 260, 64))) == ALIGN
    assert rope_call(q=heads(strides=(76800, -256, 64))) == SHAPE and rope_call(q=heads(strides=(1 << 45, 256, 64))) == SHAPE
    # the grid: tokens past its end, no extent, pairs that do not fit or make no whole vector
    assert rope_call(first=1) == SHAPE and rope_call(first=-1) == SHAPE and rope_call(r=rope(extent=(3, 0, 10))) == SHAPE
    assert rope_call(r=rope(extent=(1 << 31, 1, 1))) == SHAPE and rope_call(r=rope(extent=(65536, 32768, 2))) == SHAPE
    for bad in ((8, 12, 16), (0, 0, 0), (1, 1, 1), (-4, 4, 4), (33, 0, 3)):
        assert rope_call(r=rope(pairs=bad)) == SHAPE, bad
    for bad in (dict(theta=0.0), dict(theta=-1.0), dict(theta=math.inf), dict(theta=math.nan), dict(layout=2), dict(norm_eps=math.nan),
                dict(norm_eps=math.inf), dict(origin=(math.nan, 0, 0)), dict(origin=(0, 2e12, 0)), dict(step=(1, 1, math.inf)), dict(step=(1e12, 1, 1))):
        assert rope_call(r=rope(**bad)) == ARG, bad
    assert rope_call(r=rope(norm_eps=1e-6, q_gain=BASE + 2)) == ALIGN and rope_call(r=rope(norm_eps=1e-6, k_gain=BASE + 8)) == ALIGN


def test_rope_operands_that_overlap():
    wide = (300 * 768, 768, 64)  # q | k | v in rows of 12 heads
    q, k = heads(strides=wide), heads(256 * 2, strides=wide)
    # an output between the rows of an input, but on its elements
    assert rope_call(q=q, k=k, qo=heads(64 * 2, strides=wide), ko=heads(FAR)) == ARG
    # both outputs in one place, one's input under the other's output
    assert rope_call(qo=heads(2 * FAR), ko=heads(2 * FAR)) == ARG
    assert rope_call(q=heads(), k=heads(FAR), qo=heads(FAR), ko=heads(2 * FAR)) == ARG
    # in place, but with other strides or shifted
    assert rope_call(qo=heads(64 * 2)) == ARG
    # an output whose elements share addresses
    for s in ((0, 256, 64), (76800, 0, 64), (76800, 256, 0), (76800, 256, 32), (256, 256, 64)):
        assert rope_call(qo=heads(2 * FAR, strides=s)) == ARG, s


def select(q=None, k=None, q_block=64, k_block=64, keep=3, q_len=None, k_len=None, blocks=BITS, ws=WS, nbytes=1 << 40):
    q, k = q or heads(), k or heads(FAR)
    return si.lib().si_attn_select(C.byref(q), C.byref(k), q_block, k_block, keep, q_len, k_len, blocks, ws, nbytes, None)


def sparse(q=None, k=None, v=None, q_block=64, k_block=64, scale=0.125, q_len=None, k_len=None, blocks=BITS, out=None, ws=WS, nbytes=1 << 40):
    q, k, v, out = q or heads(), k or heads(FAR), v or heads(2 * FAR), out or heads(3 * FAR)
    return si.lib().si_attn_sparse_forward(C.byref(q), C.byref(k), C.byref(v), q_block, k_block, scale, q_len, k_len, blocks, C.byref(out), ws, nbytes, None)


@pytest.mark.parametrize("call", [select, sparse])
def test_runs_and_blocks_refusals(call):
    for bad in (dict(q_block=0), dict(q_block=-1), dict(q_block=1 << 21), dict(k_block=0), dict(k_block=32), dict(k_block=96), dict(k_block=1 << 21)):
        assert call(**bad) == SHAPE, bad
    assert call(q=heads(H=6)) == SHAPE                       # 6 query heads on 4 key heads
    assert call(k=heads(FAR, Bn=1)) == SHAPE and call(k=heads(FAR, d=32)) == SHAPE and call(k=heads(FAR, dtype=B.SI_F32)) == DTYPE
    assert call(k=heads(FAR, strides=(1 << 34, 1 << 23, 64))) == SHAPE
    assert call(q=heads(ptr=0)) == NULL and call(ws=None) == NULL
    assert call(ws=WS + 16) == ALIGN and call(blocks=BITS + 2) == ALIGN and call(q_len=LEN + 1) == ALIGN and call(k_len=LEN + 2) == ALIGN
    assert call(nbytes=16) == WORKSPACE
    assert call(ws=BASE) == ARG and call(ws=BASE + FAR) == ARG                     # workspace on an operand
    assert call(q_len=WS) == ARG and call(k_len=WS) == ARG                        # lengths in the workspace
    # more lists than 32 bits count
    many = dict(Bn=1 << 12, N=1 << 20, strides=(1 << 26, 64, 64), H=1)
    assert call(q=heads(**many), k=heads(FAR * 1024, **many), q_block=1) == SHAPE


def test_selection_refusals():
    assert select(keep=0) == ARG and select(keep=-5) == ARG
    assert select(blocks=None) == NULL and select(blocks=BASE + 4096) == ARG and select(blocks=WS) == ARG
    long = heads(FAR, N=64 * 16384 + 1, Bn=1)
    assert select(q=heads(Bn=1), k=long) == SHAPE
    assert select(q=heads(Bn=1), k=heads(FAR, N=64 * 16384, Bn=1), nbytes=16) == WORKSPACE   # the longest that is taken


def test_attention_refusals():
    for bad in (0.0, -1.0, math.nan, math.inf):
        assert sparse(scale=bad) == ARG, bad
    assert sparse(v=heads(2 * FAR, N=299)) == SHAPE and sparse(v=heads(2 * FAR, dtype=B.SI_F32)) == DTYPE
    assert sparse(v=heads(2 * FAR, strides=(1 << 34, 1 << 23, 64))) == SHAPE
    assert sparse(out=heads(3 * FAR, H=5)) == SHAPE and sparse(out=heads(3 * FAR, dtype=B.SI_F32)) == DTYPE
    assert sparse(out=heads()) == ARG and sparse(out=heads(FAR)) == ARG and sparse(out=heads(2 * FAR + 4096)) == ARG
    assert sparse(out=heads(3 * FAR, strides=(76800, 0, 64))) == ARG
    assert sparse(blocks=BASE + 3 * FAR) == ARG and sparse(blocks=WS) == ARG
    # 64 times the key heads' stride: one token that is split over many workgroups needs its workspace
    one, cache = heads(N=1, H=32, Bn=1), heads(FAR, N=100000, H=8, Bn=1)
    need = si.lib().si_attn_sparse_workspace_bytes(C.byref(one), C.byref(cache), 1, 64)
    assert need > 1 << 16
    assert sparse(q=one, k=cache, v=heads(2 * FAR, N=100000, H=8, Bn=1), q_block=1, out=heads(3 * FAR, N=1, H=32, Bn=1), nbytes=need - 1) == WORKSPACE


def test_workspace_and_word_counts():
    by = C.byref
    assert si.si_attn_block_words(0, 64) == 0 and si.si_attn_block_words(1, 64) == 1 and si.si_attn_block_words(64 * 32 + 1, 64) == 2
    assert si.si_attn_block_words(-1, 64) == 0 and si.si_attn_block_words(100, 65) == 0 and si.si_attn_block_words(100, 0) == 0
    for fn in (si.lib().si_attn_select_workspace_bytes, si.lib().si_attn_sparse_workspace_bytes):
        assert fn(by(heads()), by(heads(FAR)), 64, 64) > 0
        assert fn(by(heads(d=20)), by(heads(FAR)), 64, 64) == 0 and fn(by(heads()), by(heads(FAR)), 64, 100) == 0


def test_block_refusals():
    x = B._Tensor5(BASE, B.SI_BF16, 2, 64, 4, 8, 8)
    out = B._Tensor5(BASE + FAR, B.SI_BF16, 2, 64, 4, 8, 8)
    ctx = B._Context(BASE + 2 * FAR, B.SI_BF16, 2, 5, 16)

    def weights(kind):
        w = B._Weights()
        w.kind, w.heads, w.dim_head, w.gn_groups, w.gn_eps, w.ln_eps, w.add_sin_pe = kind, 2, 32, 8, 1e-6, 1e-5, 0
        for name in B.WEIGHT_FIELDS:
            setattr(w, name, BASE + 3 * FAR)
        return w

    def call(attn, kind=B.SI_BLOCK_SPATIAL, axis=B.SI_AXIS_F, flags=0, nbytes=1 << 40):
        return si.lib().si_block_forward_attn(C.byref(x), C.byref(weights(kind)), C.byref(ctx), None if attn is None else C.byref(attn.struct),
                                              C.byref(out), axis, 1, WS, nbytes, flags, None)

    def size(attn, kind=B.SI_BLOCK_SPATIAL, axis=B.SI_AXIS_F):
        return si.lib().si_block_attn_workspace_bytes(C.byref(x), C.byref(weights(kind)), C.byref(ctx), C.byref(attn.struct), axis, 1)

    good = si.AttnOptions(si.Rope((4, 8, 8), (4, 4, 8)), q_block=32, k_block=64, keep=1)
    assert size(good) > 0 and call(good, nbytes=64) == WORKSPACE
    assert call(None) == NULL and call(good, flags=2) == ARG
    assert call(good, kind=B.SI_BLOCK_TEMPORAL, axis=B.SI_AXIS_HW) == ARG and size(good, kind=B.SI_BLOCK_TEMPORAL, axis=B.SI_AXIS_HW) == 0
    assert call(good, axis=B.SI_AXIS_HW) == SLICE
    assert call(si.AttnOptions(keep=-1)) == ARG
    for bad in (dict(q_block=0), dict(k_block=63), dict(k_block=0)):
        assert call(si.AttnOptions(keep=1, **bad)) == SHAPE and size(si.AttnOptions(keep=1, **bad)) == 0
    assert call(si.AttnOptions(si.Rope((4, 8, 9), (4, 4, 8)))) == SHAPE               # another map than the block's
    assert call(si.AttnOptions(si.Rope((4, 8, 8), (4, 4, 12)))) == SHAPE              # more pairs than a head has
    assert call(si.AttnOptions(si.Rope((4, 8, 8), (4, 4, 8), theta=0.0))) == ARG
    # what the block without options needs does not change with them
    base = si.lib().si_workspace_bytes(C.byref(x), C.byref(weights(B.SI_BLOCK_SPATIAL)), C.byref(ctx), B.SI_AXIS_F, 1)
    assert size(si.AttnOptions()) == base and size(good) > base


def test_binding_refuses_what_it_cannot_describe():
    x = torch.zeros(1, 4, 2, 64)
    r = si.Rope((1, 2, 2), (0, 8, 8))
    with pytest.raises(ValueError):
        si.si_rope_forward(x, None, r, x.clone(), None)                                # not on a GPU
    with pytest.raises(ValueError):
        si.si_rope_forward(x[0], None, r, x.clone(), None)
    with pytest.raises(ValueError):
        si.si_rope_forward(x.transpose(2, 3), None, r, x.clone(), None)
    with pytest.raises(ValueError):
        si.Rope((1, 2, 2), (0, 8, 8), q_gain=torch.zeros(64))                          # a gain without the norm
    with pytest.raises(ValueError):
        si.Rope((1, 2, 2), (0, 8, 8), norm_eps=-1.0)
    with pytest.raises(ValueError):
        si.si_rope_forward(x, None, si.Rope((1, 2, 2), (0, 8, 8), norm_eps=1e-6, q_gain=torch.zeros(32)), x.clone(), None)
    words = torch.zeros(1, 2, 1, 1, dtype=torch.int32)
    ws = torch.zeros(1 << 16, dtype=torch.uint8)
    for bad in (words.long(), words[0], torch.zeros(1, 2, 1, 2, dtype=torch.int32), torch.zeros(1, 2, 2, 1, dtype=torch.int32)[:, :, ::2]):
        with pytest.raises(ValueError):
            si.si_attn_select(x, x, 4, 64, 1, bad, ws)
    for bad in (torch.zeros(2, dtype=torch.int32), torch.zeros(1, dtype=torch.int64)):
        with pytest.raises(ValueError):
            si.si_attn_sparse_forward(x, x, x, 4, 64, words, x.clone(), ws, k_len=bad)
    with pytest.raises(si.SiError):
        si.si_attn_select(x, x, 0, 64, 1, words, ws)


def test_gains_under_an_output():
    """A gain that the call would overwrite while other workgroups read it."""
    size = 2 * 300 * 4 * 64 * 2
    for at in (2 * FAR, 2 * FAR + size - 128, 3 * FAR + 4096):
        for name in ("q_gain", "k_gain"):
            assert rope_call(r=rope(norm_eps=1e-6, **{name: BASE + at})) == ARG, (at, name)
    x, out = B._Tensor5(BASE, B.SI_BF16, 2, 64, 4, 8, 8), B._Tensor5(BASE + FAR, B.SI_BF16, 2, 64, 4, 8, 8)
    ctx = B._Context(BASE + 2 * FAR, B.SI_BF16, 2, 5, 16)
    w = B._Weights()
    w.kind, w.heads, w.dim_head, w.gn_groups, w.gn_eps, w.ln_eps, w.add_sin_pe = B.SI_BLOCK_SPATIAL, 2, 32, 8, 1e-6, 1e-5, 0
    for name in B.WEIGHT_FIELDS:
        setattr(w, name, BASE + 3 * FAR)
    for gain in (WS + 1024, BASE + FAR + 64):
        r = rope(pairs=(4, 4, 8), extent=(4, 8, 8), norm_eps=1e-6, k_gain=gain)
        attn = B._AttnOptions(C.pointer(r), 32, 64, 1)
        assert si.lib().si_block_forward_attn(C.byref(x), C.byref(w), C.byref(ctx), C.byref(attn), C.byref(out), B.SI_AXIS_F, 1, WS, 1 << 40,
                                              0, None) == ARG


def test_angles_and_scales_that_float_cannot_hold():
    assert rope_call(r=rope(theta=1e-3, origin=(2e9, 0, 0))) == ARG and rope_call(r=rope(theta=1e-3, step=(1, 2e8, 1))) == ARG
    assert rope_call(r=rope(theta=5e-324)) == ARG
    assert sparse(scale=3e38) == ARG


# ------------------------------------------------------------------------------------------------ the oracle

def test_oracle_rotation_is_relative_and_keeps_lengths():
    """Rotated inner products depend on the distance of the positions only, per axis; norms do not change."""
    rng = np.random.default_rng(0)
    pairs, d = (3, 4, 5), 28
    a, b = rng.standard_normal((2, 1, 1, 1, d))
    for halves in (False, True):
        dots = {}
        for origin in ((0, 0, 0), (5, -2, 9)):
            ang = oracle.rope_angles_ref((2, 3, 4), pairs, 30.0, origin)
            xa = np.concatenate([oracle.rope_ref(a, ang[n:n + 1], halves) for n in range(24)], axis=1)[0, :, 0]
            xb = np.concatenate([oracle.rope_ref(b, ang[n:n + 1], halves) for n in range(24)], axis=1)[0, :, 0]
            dots[origin] = xa @ xb.T
            assert np.allclose((xa ** 2).sum(-1), (a ** 2).sum())
        assert np.allclose(dots[(0, 0, 0)], dots[(5, -2, 9)])
        assert not np.allclose(dots[(0, 0, 0)][0], dots[(0, 0, 0)][0, 0])
    # by hand: one pair, a quarter turn at position 1 where theta^0 * step = pi / 2
    y = oracle.rope_ref(np.array([[[[1.0, 2.0, 7.0]], [[1.0, 2.0, 7.0]]]]), oracle.rope_angles_ref((1, 1, 2), (0, 0, 1), step=(1, 1, math.pi / 2)))
    assert np.allclose(y[0, :, 0], [[1, 2, 7], [-2, 1, 7]])


def test_oracle_selection_and_attention_by_hand():
    k = np.zeros((1, 200, 1, 8))
    k[0, 64:128, 0, 0], k[0, 128:192, 0, 0], k[0, 192:, 0, 0] = 1.0, 3.0, 2.0
    q = np.zeros((1, 3, 2, 8))
    q[..., 0] = [[1, 3], [1, 1], [-1, -1]]
    s = oracle.block_scores_ref(q, k, 2, 64)
    assert np.allclose(s[0, 0], [[0, 1.5, 4.5, 3], [0, -1, -3, -2]])
    kept = oracle.select_ref(q, k, 2, 64, 2)
    assert kept[0, 0].tolist() == [[False, False, True, True], [True, True, False, False]]
    assert oracle.pack_blocks_ref(kept).tolist() == [[[[12], [3]]]]
    assert oracle.pack_blocks_ref(np.arange(40)[None] == 31).tolist() == [[-(1 << 31), 0]]
    v = np.arange(200.0).reshape(1, 200, 1, 1) * np.ones(8)
    out, spread, mass = oracle.sparse_attention_ref(q * 0, k, v, kept, 2, 64)
    assert np.allclose(out[0, 0], np.mean(np.arange(128, 200))) and np.allclose(out[0, 2], np.mean(np.arange(128)))
    assert np.allclose(mass, out) and np.allclose(spread[0, 0], np.mean(np.abs(np.arange(128, 200) - 163.5)))


def test_oracle_block_without_options_is_the_plain_block():
    spec = wl.BlockSpec("b", wl.SPATIAL, "f32", 1, 16, 2, 6, 12, 2, 8, gn_groups=4, ctx_tokens=3, ctx_dim=8, slice_axis=wl.AXIS_F, slice_len=1, seed=3)
    x, w, ctx = wl.make_x(spec), wl.make_weights(spec, randomize_affine=True, matrix_std=0.3), wl.make_context(spec)
    plain = oracle.block_forward_ref(x, w, spec, ctx)
    assert np.allclose(oracle.block_forward_attn_ref(x, w, spec, ctx), plain, rtol=0, atol=1e-12)
    assert np.allclose(oracle.block_forward_attn_ref(x, w, spec, ctx, keep=2), plain, rtol=0, atol=1e-12)
    assert not np.allclose(oracle.block_forward_attn_ref(x, w, spec, ctx, keep=1), plain, atol=1e-4)


def test_block_without_lists_takes_any_sizes_of_runs_and_blocks():
    x = B._Tensor5(BASE, B.SI_BF16, 2, 64, 4, 8, 8)
    ctx = B._Context(BASE + 2 * FAR, B.SI_BF16, 2, 5, 16)
    w = B._Weights()
    w.kind, w.heads, w.dim_head, w.gn_groups, w.gn_eps, w.ln_eps, w.add_sin_pe = B.SI_BLOCK_SPATIAL, 2, 32, 8, 1e-6, 1e-5, 0
    size = lambda **kw: si.lib().si_block_attn_workspace_bytes(C.byref(x), C.byref(w), C.byref(ctx), C.byref(si.AttnOptions(**kw).struct), B.SI_AXIS_F, 1)  # noqa: E731
    assert size() > 0
    for sizes in ((0, 0), (-1, 7), (1 << 40, 1 << 40), (1, 64)):
        assert size(q_block=sizes[0], k_block=sizes[1], keep=0) == size(), sizes
        assert size(q_block=sizes[0], k_block=sizes[1], keep=1) == 0 or sizes == (1, 64)


def test_word_counts_of_sizes_that_no_call_takes():
    most = 2 ** 31 - 1 - 2 ** 22  # tokens of a sequence
    assert si.si_attn_block_words(most, 64) == -(-most // 2048) and si.si_attn_block_words(most, 1 << 20) == 64
    for n_keys, k_block in ((most + 1, 64), (2 ** 63 - 1, 64), (2 ** 63 - 1, 1 << 20), (100, (1 << 20) + 64), (100, 1 << 40), (100, -64)):
        assert si.si_attn_block_words(n_keys, k_block) == 0, (n_keys, k_block)


def test_frequencies_that_double_cannot_hold():
    """theta^(-i / pairs) of a subnormal theta is infinite, and zero times it no angle."""
    still = dict(origin=(0, 0, 0), step=(0, 0, 0))
    q = heads(N=1 << 30)  # behind the grid: what is no refusal of theta is this one, before any launch
    for theta, want in ((1e-310, ARG), (5e-324, ARG), (2.3e-308, SHAPE), (1e308, SHAPE)):
        assert rope_call(q=q, qo=heads(2 * FAR, N=1 << 30), lone=True, r=rope(theta=theta, **still)) == want, theta
