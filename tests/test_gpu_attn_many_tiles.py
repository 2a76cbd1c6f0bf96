"""More row tiles and runs than a launch has workgroups (2^20): every workgroup takes several, one after the other.  A small
set of queries stands in the call many times over, and every repetition has to have the bits of the small call."""
import pytest
import torch

import paper_2411_01171_amd as si

pytestmark = pytest.mark.gpu

BASE = 4096  # queries of the small call: enough row tiles that no list is dealt out


def _operands(dtype, heads, keys):
    gen = torch.Generator(device="cuda").manual_seed(heads + keys)
    draw = lambda *shape: torch.randn(*shape, generator=gen, device="cuda").to(dtype)  # noqa: E731
    return draw(1, BASE, heads, 8), draw(1, keys, 1, 8), draw(1, keys, 1, 8)


def _repeat(x, times, dim=1):
    return x.repeat([times if i == dim else 1 for i in range(x.dim())])


@pytest.mark.parametrize("dtype,heads", [(torch.bfloat16, 1), (torch.bfloat16, 40), (torch.bfloat16, 100),   # 32, 64 and 128 rows of a tile
                                         (torch.float32, 1), (torch.float32, 20), (torch.float32, 40), (torch.float32, 100)])
def test_attention(dtype, heads):
    """Runs of one token and `heads` query heads, lists of none to three blocks; the last tokens do not count."""
    times, keys = 300, 130
    q, k, v = _operands(dtype, heads, keys)
    words = torch.randint(0, 8, (1, 1, BASE, 1), dtype=torch.int32, device="cuda")
    ws = torch.empty(si.si_attn_sparse_workspace_bytes(q, k, 1, 64), dtype=torch.uint8, device="cuda")
    ref = torch.full_like(q, 7.0)
    si.si_attn_sparse_forward(q, k, v, 1, 64, words, ref, ws)
    assert torch.isfinite(ref).all() and ref.float().std() > 0.05
    many = _repeat(q, times)
    out = torch.full_like(many, 7.0)
    ws = torch.empty(si.si_attn_sparse_workspace_bytes(many, k, 1, 64), dtype=torch.uint8, device="cuda")
    q_len = torch.tensor([times * BASE - 5], dtype=torch.int32, device="cuda")
    si.si_attn_sparse_forward(many, k, v, 1, 64, _repeat(words, times, 2), out, ws, q_len=q_len)
    got = out.view(times, BASE, heads, 8)
    assert torch.equal(got[:-1], ref.expand(times - 1, -1, -1, -1))
    assert torch.equal(got[-1, :-5], ref[0, :-5]) and (got[-1, -5:] == 7).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("blocks,keep", [(4, 2), (70, 35)])
def test_selection(dtype, blocks, keep):
    """2^24 runs and more: over 2^20 tiles of sixteen."""
    times = 4200
    q, k, _ = _operands(dtype, 1, 64 * blocks - 3)
    n_words = si.si_attn_block_words(k.shape[1], 64)
    ref = torch.zeros(1, 1, BASE, n_words, dtype=torch.int32, device="cuda")
    si.si_attn_select(q, k, 1, 64, keep, ref, torch.empty(si.si_attn_select_workspace_bytes(q, k, 1, 64), dtype=torch.uint8, device="cuda"))
    bits = sum((ref >> i) & 1 for i in range(32)).sum(dim=-1)
    assert (bits == keep).all()
    many = _repeat(q, times)
    out = torch.zeros(1, 1, times * BASE, n_words, dtype=torch.int32, device="cuda")
    si.si_attn_select(many, k, 1, 64, keep, out, torch.empty(si.si_attn_select_workspace_bytes(many, k, 1, 64), dtype=torch.uint8, device="cuda"))
    assert torch.equal(out.view(times, BASE, n_words), ref[0].expand(times, -1, -1))
