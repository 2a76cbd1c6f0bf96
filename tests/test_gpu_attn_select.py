"""si_attn_select against the float64 oracle, bit for bit."""
import numpy as np
import pytest
import torch

import oracle
import paper_2411_01171_amd as si
from attn_helpers import LAYOUTS, draw, lengths, strided
from gpu_helpers import guarded, guards_intact

pytestmark = pytest.mark.gpu


def _select(dq, dk, q_block, k_block, keep, q_len=None, k_len=None, stream=None):
    B, N, _, _ = dq.shape
    Nk, Hk = dk.shape[1], dk.shape[2]
    words = si.si_attn_block_words(Nk, k_block)
    n = si.si_attn_select_workspace_bytes(dq, dk, q_block, k_block)
    assert n > 0
    ws_buf, ws = guarded(n)
    out_buf, out = guarded(torch.empty(B, Hk, -(-N // q_block), words, dtype=torch.int32))
    si.si_attn_select(dq, dk, q_block, k_block, keep, out, ws, q_len=lengths(q_len), k_len=lengths(k_len), stream=stream)
    torch.cuda.synchronize()
    assert guards_intact(ws_buf, n) and guards_intact(out_buf, out.numel() * 4)
    return out.cpu().numpy()


def _check(dtype, B, N, Nk, Hq, Hk, d, q_block, k_block, keep, q_len=None, k_len=None, layout="rows", seed=0):
    rng = np.random.default_rng(seed)
    q, k = draw(rng, (B, N, Hq, d), dtype), draw(rng, (B, Nk, Hk, d), dtype)
    dq, dk = strided(q, dtype, layout), strided(k, dtype, layout)
    for b in range(B):  # what does not count may hold anything
        if q_len is not None:
            dq[b, min(max(q_len[b], 0), N):] = float("nan")
        if k_len is not None:
            dk[b, min(max(k_len[b], 0), Nk):] = float("inf")
    got = _select(dq, dk, q_block, k_block, keep, q_len, k_len)
    want = oracle.pack_blocks_ref(oracle.select_ref(q, k, q_block, k_block, keep, q_len, k_len))
    assert np.array_equal(got, want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [8, 40, 64, 96, 128])
@pytest.mark.parametrize("q_block,k_block,keep", [(128, 64, 4), (33, 64, 1), (1, 128, 3), (1000, 192, 2)])
def test_blocks_of_ordinary_features(dtype, d, q_block, k_block, keep):
    _check(dtype, 2, 300, 700, 2, 2, d, q_block, k_block, keep)


@pytest.mark.parametrize("heads", [(4, 1), (6, 3), (16, 2)])
def test_heads_shared_by_queries(heads):
    _check("bf16", 1, 130, 900, heads[0], heads[1], 64, 32, 64, 5)


@pytest.mark.parametrize("layout", LAYOUTS)
def test_strides(layout):
    _check("bf16", 2, 140, 500, 3, 3, 64, 64, 64, 3, layout=layout)
    _check("f32", 2, 140, 500, 3, 3, 40, 64, 64, 3, layout=layout)


@pytest.mark.parametrize("q_len,k_len", [([0, 150, 200], [640, 0, 1]), ([1, 64, 65], [64, 65, 63]), ([-3, 999, 128], [7000, -1, 600])])
def test_padded_batches(q_len, k_len):
    _check("bf16", 3, 200, 650, 2, 1, 64, 64, 64, 3, q_len, k_len)


@pytest.mark.parametrize("blocks", [1, 31, 32, 33, 64, 65, 127, 129, 256, 257, 513, 1025, 2100])
def test_lists_of_every_length(blocks):
    """Through every size of the scores' store; one or two rows of scores per workgroup at the end."""
    _check("bf16", 1, 70, 64 * blocks - 17, 1, 1, 8, 2, 64, max(1, blocks // 3))


def test_longest_list():
    """16384 blocks, means set through runs of equal keys."""
    rng = np.random.default_rng(5)
    k = np.repeat(draw(rng, (1, 16384, 1, 8), "bf16"), 64, axis=1)
    q = draw(rng, (1, 3, 1, 8), "bf16")
    got = _select(strided(q, "bf16", "rows"), strided(k, "bf16", "rows"), 1, 64, 5000)
    s = np.asarray(q[0, :, 0], np.float64) @ np.asarray(k[0, ::64, 0], np.float64).T
    kept = np.zeros((1, 1, 3, 16384), bool)
    for i in range(3):
        kept[0, 0, i, np.lexsort((np.arange(16384), -s[i]))[:5000]] = True
    assert np.array_equal(got, oracle.pack_blocks_ref(kept))


def test_ties_go_to_the_lowest_block():
    q = np.ones((1, 4, 1, 8), np.float32)
    k = np.zeros((1, 64 * 40, 1, 8), np.float32)
    for j, value in ((3, 2.0), (7, 1.0), (11, 1.0), (12, -0.0), (30, 1.0), (39, -1.0)):
        k[0, 64 * j:64 * j + 64] = value
    for keep, want in ((1, {3}), (2, {3, 7}), (3, {3, 7, 11}), (5, {3, 7, 11, 30, 0}), (7, {3, 7, 11, 30, 0, 1, 2}), (39, set(range(39))), (99, set(range(40)))):
        for dtype in ("bf16", "f32"):
            got = _select(strided(q, dtype, "rows"), strided(k, dtype, "rows"), 4, 64, keep)
            kept = np.array([[[[j in want for j in range(40)]]]])
            assert np.array_equal(got, oracle.pack_blocks_ref(kept)), keep


def test_scores_that_differ_in_the_last_digits_only():
    """Means 1 + j 2^-30 (bf16 values 1 and small ones in 64 rows): the order is that of float64, not of float32."""
    q = np.ones((1, 1, 1, 8), np.float32)
    k = np.zeros((1, 64 * 20, 1, 8), np.float32)
    order = np.random.default_rng(3).permutation(20)
    for j in range(20):
        k[0, 64 * j:64 * j + 64, 0, 0] = 1.0
        k[0, 64 * j, 0, 1] = order[j] * 2.0 ** -24
    for keep in (1, 5, 19):
        got = _select(strided(q, "bf16", "rows"), strided(k, "bf16", "rows"), 1, 64, keep)
        assert np.array_equal(got, oracle.pack_blocks_ref((order >= 20 - keep)[None, None, None]))


@pytest.mark.parametrize("kind", ["wide", "negative", "one_far_above", "one_upper_word", "equal", "two_values"])
@pytest.mark.parametrize("blocks", [20, 50, 100, 200, 400, 1000, 1500])
def test_distributions_of_scores(kind, blocks):
    """Blocks of equal keys (value, 0, ...) against queries (1, 0, ...), (-1, 0, ...) and (2, 0, ...): scores known exactly."""
    rng = np.random.default_rng(blocks)
    value = {"wide": rng.standard_normal(blocks) * 2.0 ** rng.integers(-60, 60, blocks),
             "negative": -1 - rng.random(blocks),
             "one_far_above": np.where(np.arange(blocks) == blocks // 2, 1e30, rng.standard_normal(blocks)),
             "one_upper_word": 1 + rng.integers(0, 8, blocks) * 2.0 ** -23,  # float64's upper 32 bits agree
             "equal": np.full(blocks, 0.75),
             "two_values": rng.integers(0, 2, blocks) * 1.0}[kind].astype(np.float32)
    k = np.zeros((1, blocks * 64, 1, 8), np.float32)
    k[0, :, 0, 0] = np.repeat(value, 64)
    q = np.zeros((1, 3, 1, 8), np.float32)
    q[0, :, 0, 0] = 1, -1, 2
    dq, dk = strided(q, "f32", "rows"), strided(k, "f32", "rows")
    for keep in (1, blocks // 3, blocks - 1):
        kept = np.zeros((1, 1, 3, blocks), bool)
        for i in range(3):
            kept[0, 0, i, np.lexsort((np.arange(blocks), -(value.astype(np.float64) * q[0, i, 0, 0])))[:keep]] = True
        assert np.array_equal(_select(dq, dk, 1, 64, keep), oracle.pack_blocks_ref(kept)), keep


def test_scores_that_are_not_finite():
    q = np.ones((1, 1, 1, 8), np.float32)
    k = np.zeros((1, 64 * 6, 1, 8), np.float32)
    k[0, 0], k[0, 64], k[0, 128, 0, 0], k[0, 192, 0, 0], k[0, 192, 0, 1] = np.nan, -np.inf, np.inf, np.inf, -np.inf
    k[0, 256] = 5.0
    got = [_select(strided(q, "f32", "rows"), strided(k, "f32", "rows"), 1, 64, keep) for keep in (1, 2, 3, 4, 5)]
    want = ({2}, {2, 4}, {2, 4, 5}, {0, 2, 4, 5}, {0, 1, 2, 4, 5})
    for g, w in zip(got, want):
        assert np.array_equal(g, oracle.pack_blocks_ref(np.array([[[[j in w for j in range(6)]]]])))


def test_no_keys_and_no_queries():
    q, k = torch.randn(2, 5, 2, 64, device="cuda"), torch.randn(2, 100, 2, 64, device="cuda")
    assert _select(q, k[:, :0], 4, 64, 2).size == 0
    assert _select(q[:, :0], k, 4, 64, 2).size == 0


def test_captured_call_replays_like_the_eager_one():
    q, k = torch.randn(1, 256, 4, 64, device="cuda"), torch.randn(1, 2000, 2, 64, device="cuda")
    ws = torch.empty(si.si_attn_select_workspace_bytes(q, k, 64, 64), dtype=torch.uint8, device="cuda")
    ref, out = (torch.zeros(1, 2, 4, 1, dtype=torch.int32, device="cuda") for _ in range(2))
    si.si_attn_select(q, k, 64, 64, 7, ref, ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        si.si_attn_select(q, k, 64, 64, 7, out, ws)
    for i in range(3):
        q.normal_()
        si.si_attn_select(q, k, 64, 64, 7, ref, ws)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, ref), i


@pytest.mark.parametrize("blocks,keep", [(70, 35), (72, 36), (80, 60), (129, 65), (144, 72), (300, 200), (900, 450)])
def test_many_of_the_blocks_kept_in_full_tiles_of_runs(blocks, keep):
    """Thresholds far below the largest score, sixteen runs to a workgroup whose scores lie next to each other."""
    _check("bf16", 1, 48, 64 * blocks - 5, 2, 2, 8, 1, 64, keep, seed=blocks)


@pytest.mark.parametrize("blocks,counted,keep", [(100, 70, 40), (300, 60, 30), (500, 70, 66), (900, 100, 80)])
def test_padded_batches_of_long_lists(blocks, counted, keep):
    """Most of the places of a list stand for blocks without a counted key."""
    _check("f32", 2, 40, 64 * blocks, 1, 1, 8, 1, 64, keep, q_len=[40, 33], k_len=[64 * counted - 3, 64 * blocks], seed=blocks)
