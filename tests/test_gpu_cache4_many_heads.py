"""Calls on the cache in 4 bits with more heads than a launch has workgroups: every one is walked to the end."""
import numpy as np
import pytest
import torch

import paper_2411_01171_amd as si

pytestmark = pytest.mark.gpu

B, H, CAP, D = 1030, 1024, 4, 8  # 1 054 720 heads, a launch has 1 048 576 workgroups at most


def test_store_attend_and_evict():
    gen = torch.Generator(device="cuda").manual_seed(1)
    # small whole numbers of which a 6 is the largest: stored exactly
    whole = lambda *shape: torch.tensor([0, 1, -1, 2, -2, 3, 4, -4], device="cuda")[torch.randint(0, 8, shape, generator=gen, device="cuda")].to(torch.bfloat16)  # noqa: E731
    k, v, q = whole(B, CAP, H, D), whole(B, CAP, H, D), whole(B, 1, H, D)
    k[..., 0], v[..., 0] = 6, 6
    cache = si.Cache4.empty(B, H, CAP, D)
    si.si_cache4_store(k, v, cache)
    ko, vo = torch.empty_like(k), torch.empty_like(v)
    si.si_cache4_load(cache, ko, vo)
    assert torch.equal(ko, k) and torch.equal(vo, v)

    out, weight = torch.empty_like(q), torch.empty(B, H, CAP, device="cuda")
    ws = torch.empty(si.si_cache4_attn_workspace_bytes(q, cache, True), dtype=torch.uint8, device="cuda")
    si.si_cache4_attn_forward(q, cache, out, ws, scale=0.125, weight_out=weight)
    s = (q.double() * k.double()).sum(dim=-1).transpose(1, 2) * 0.125       # [B, H, CAP]; exact in float32 too
    p = torch.softmax(s, dim=-1)
    ref = (p.transpose(1, 2).unsqueeze(-1) * v.double()).sum(dim=1, keepdim=True)
    # two weights of rounded exponentials each (exp2 to 2^-22, 24 bits of the exponent's fma), a sum of four, a division
    assert bool(((weight.double() - p).abs() <= p * (2 * 2.0 ** -22 + 2 * 24 * 2.0 ** -24 + 8 * 2.0 ** -24)).all())
    # weights rounded to bf16 (half a step of 2^-8), |v - out| up to 12; the output's own rounding
    assert bool(((out.double() - ref).abs() <= 2.0 ** -8 * 1.01 * (12 + ref.abs())).all())

    keep = 2
    less = si.Cache4.empty(B, H, keep, D)
    w_out, kept, n = torch.empty(B, H, keep, device="cuda"), torch.empty(B, H, keep, dtype=torch.int32, device="cuda"), torch.empty(B, dtype=torch.int32, device="cuda")
    ws = torch.empty(si.si_cache4_evict_workspace_bytes(cache, keep), dtype=torch.uint8, device="cuda")
    si.si_cache4_evict(cache, weight, keep, less, w_out, kept, n, ws)
    at = weight.argsort(dim=-1, descending=True, stable=True)[..., :keep].sort(dim=-1).values
    assert torch.equal(kept.long(), at) and bool((n == keep).all()) and torch.equal(w_out, weight.gather(-1, at))
    for got, all_of in zip(less.tensors, cache.tensors):
        assert torch.equal(got, all_of.gather(2, at.unsqueeze(-1).expand(-1, -1, -1, all_of.shape[-1])))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_queries_by_the_hundred(dtype):
    """Tiles of many rows (bf16: 128), and more of them than workgroups: some heads against calls of their own."""
    gen = torch.Generator(device="cuda").manual_seed(2)
    b, n, h = B, 70, H
    q = torch.randn(b, n, h, 8, generator=gen, device="cuda", dtype=dtype)
    cache = si.Cache4(*(torch.randint(0, 256, (b, h, 40, c), generator=gen, device="cuda", dtype=torch.uint8) if c == 16
                        else torch.full((b, h, 40, 1), 126, device="cuda", dtype=torch.uint8) for c in (16, 1, 16, 1)), 8)
    for t in (cache.k_codes, cache.v_codes):
        t[..., 4:] = 0
    out, weight = torch.empty_like(q), torch.empty(b, h, 40, device="cuda")
    ws = torch.empty(si.si_cache4_attn_workspace_bytes(q, cache, True), dtype=torch.uint8, device="cuda")
    si.si_cache4_attn_forward(q, cache, out, ws, weight_out=weight)
    for at in (0, 1, h // 2, h - 2, h - 1):
        part = si.Cache4(*(t[:, at:at + 1].contiguous() for t in cache.tensors), 8)
        o, w = torch.empty(b, n, 1, 8, device="cuda", dtype=dtype), torch.empty(b, 1, 40, device="cuda")
        ws = torch.empty(si.si_cache4_attn_workspace_bytes(o, part, True), dtype=torch.uint8, device="cuda")
        si.si_cache4_attn_forward(q[:, :, at:at + 1].contiguous(), part, o, ws, weight_out=w)
        assert torch.equal(o, out[:, :, at:at + 1]) and torch.equal(w, weight[:, at:at + 1]), at
