"""Eviction from lists that several workgroups search: more than eight of them, and pieces of more than one batch."""
import pytest
import torch

import paper_2411_01171_amd as si
from attn_helpers import lengths
from gpu_helpers import guarded, guards_intact

pytestmark = pytest.mark.gpu


def _reference(w, keep, first, last, n):
    """Slots that stay of lists [lists, cap] of which n[list] count, ascending; cap where there is none."""
    lists, cap = w.shape
    j, n = torch.arange(cap, device="cuda"), n.view(-1, 1)
    rank = torch.where(j >= n, 0, torch.where((j < first) | (j >= n - last), 2, 1))
    by_weight = torch.where(w.isnan(), -float("inf"), w).argsort(dim=-1, descending=True, stable=True)
    order = by_weight.gather(-1, rank.gather(-1, by_weight).argsort(dim=-1, descending=True, stable=True))[:, :keep]
    at = torch.arange(keep, device="cuda")
    return torch.where(at < n, order, cap).sort(dim=-1).values


@pytest.mark.parametrize("B,heads,cap,k_len", [
    (1, 3, 140000, None),                     # nine pieces
    (2, 2, 200001, [200001, 139999]),         # thirteen; the last of them empty in one list
    (1, 2, 262145, None),                     # sixteen, of two batches each, most of them empty
    (3, 1, 700003, [700003, 300000, 20]),     # of three batches
    (300, 2, 33000, None),                    # many lists: one piece of three batches
    (2, 200, 50000, [50000, 16385]),          # two pieces of two batches
])
@pytest.mark.parametrize("kind", ["random", "steps", "special"])
def test_pieces(B, heads, cap, k_len, kind):
    gen = torch.Generator(device="cuda").manual_seed(cap)
    d = 8
    w = torch.rand(B, heads, cap, generator=gen, device="cuda")
    if kind == "steps":  # ties everywhere
        w = (w * 40).floor()
    elif kind == "special":
        pick = torch.randint(0, 9, w.shape, generator=gen, device="cuda")
        w = torch.tensor([float("nan"), float("inf"), -float("inf"), 0.0, -0.0, 1e-45, 1.0, -1.0, 3e38], device="cuda")[pick]
    cache = si.Cache4(*(torch.randint(0, 256, (B, heads, cap, c), generator=gen, device="cuda", dtype=torch.uint8) for c in (16, 1, 16, 1)), d)
    n = torch.full((B,), cap, device="cuda") if k_len is None else torch.tensor(k_len, device="cuda")
    for keep, first, last in ((cap // 4, 0, 0), (cap - 1, 4, cap // 2), (1, 0, 0), (1000, 400, 600)):
        out = si.Cache4(*(torch.zeros(B, heads, keep, c, device="cuda", dtype=torch.uint8) for c in (16, 1, 16, 1)), d)
        w_out, kept = torch.zeros(B, heads, keep, device="cuda"), torch.full((B, heads, keep), cap, dtype=torch.int32, device="cuda")
        out_len = torch.zeros(B, dtype=torch.int32, device="cuda")
        size = si.si_cache4_evict_workspace_bytes(cache, keep)
        buf, ws = guarded(size)
        si.si_cache4_evict(cache, w, keep, out, w_out, kept, out_len, ws, first=first, last=last, k_len=lengths(k_len))
        torch.cuda.synchronize()
        assert guards_intact(buf, size)
        at = _reference(w.view(B * heads, cap), keep, first, last, n.repeat_interleave(heads)).view(B, heads, keep)
        assert torch.equal(kept.long(), at) and torch.equal(out_len.long(), n.clamp(max=keep))
        there, at = at < cap, at.clamp(max=cap - 1)
        want = torch.where(there, w.gather(-1, at), 0.0)
        assert torch.equal(w_out.isnan(), want.isnan()) and torch.equal(w_out.nan_to_num(0.5), want.nan_to_num(0.5))
        for got, all_of in zip(out.tensors, cache.tensors):
            want = all_of.gather(2, at.unsqueeze(-1).expand(-1, -1, -1, all_of.shape[-1])).masked_fill(~there.unsqueeze(-1), 0)
            assert torch.equal(got, want)
