"""Operators of attention over video tokens: rotary positions on three axes, the choice of key blocks by a cheap score, and
attention over the chosen blocks; sizes, inputs, the plain form, one pass and the work that it cannot do without.

A case is one call as a denoising loop makes it: queries, keys and values lie interleaved in the rows of one projection
(or in a cache), positions are those of an F x H x W latent.  Features are N(0,1), keys and queries with a part that is
common to their neighbourhood, so that block means carry information, as they do in a video.
"""
import math

import torch

own = False  # True: run() calls the library

DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------------------------------------ cases

def _rope(F, H, W, heads, d, pairs, *, B=2, kv_heads=0, dtype="bf16", layout="interleaved", norm=False, origin=0, step=1.0, theta=1e4):
    return {"op": "rope", "B": B, "F": F, "H": H, "W": W, "heads": heads, "kv_heads": kv_heads or heads, "d": d, "pf": pairs[0],
            "ph": pairs[1], "pw": pairs[2], "dtype": dtype, "layout": layout, "norm": norm, "origin": origin, "step": step, "theta": theta}


def _select(N, heads, d, q_block, k_block, keep, *, B=2, kv_heads=0, Nk=0, dtype="bf16", ragged=False):
    return {"op": "select", "B": B, "N": N, "Nk": Nk or N, "heads": heads, "kv_heads": kv_heads or heads, "d": d, "q_block": q_block,
            "k_block": k_block, "keep": keep, "dtype": dtype, "ragged": ragged}


def _attn(N, heads, d, q_block, k_block, keep, **more):
    return dict(_select(N, heads, d, q_block, k_block, keep, **more), op="attn")


def listed():
    return [dict(case, name=name) for name, case in (
        # one frame of the deepest level (16x16 map, 20 heads of 64): all latency
        ("rope_16x16", _rope(1, 16, 16, 20, 64, (0, 16, 16), B=1)),
        # one-frame window of the largest spatial block (72x128 map, 5 heads of 64), both guidance halves
        ("rope_72x128", _rope(1, 72, 128, 5, 64, (0, 16, 16))),
        # the whole 25-frame video at that level, heads normalised in the same pass, channel halves as pairs
        ("rope_video_norm", _rope(25, 72, 128, 5, 64, (8, 12, 12), layout="halves", norm=True)),
        # single precision at a ragged size, uneven axes and a part of each head left alone, far along a stream of frames,
        # positions of a larger map squeezed into the trained range
        ("rope_f32_far", _rope(14, 45, 50, 8, 80, (13, 10, 13), B=1, dtype="f32", origin=1000003, step=0.75)),
        # frames of the second level (32x32 map, 10 heads of 64), all 32 of a guided 16-frame video at once
        ("select_32x32", _select(1024, 10, 64, 128, 64, 4, B=32)),
        # 25 frames of that level attended together (36x64 map): 450 runs of queries against 900 blocks of keys
        ("select_video", _select(57600, 10, 64, 128, 64, 90)),
        # padded batch in single precision, heads of 40, short runs and a last block that is not full
        ("select_f32_padded", _select(4050, 8, 40, 32, 64, 12, B=3, dtype="f32", ragged=True)),
        # one new token against a long cache of frames: 32 query heads share 8 key / value heads
        ("attn_one_token", _attn(1, 32, 128, 1, 64, 256, B=4, kv_heads=8, Nk=115200)),
        # self-attention of the largest spatial block's one-frame window over a quarter of its keys
        ("attn_72x128", _attn(9216, 5, 64, 128, 64, 36)),
        # 25 frames of the second level attended together over a tenth of the keys: the largest call
        ("attn_video", _attn(57600, 10, 64, 128, 64, 90)),
        # single precision, 64x64 map, heads of 40
        ("attn_f32_d40", _attn(4096, 8, 40, 64, 64, 16, dtype="f32")),
        # padded batch, heads of 128 in groups, odd length, wide blocks
        ("attn_d128_padded", _attn(14999, 8, 128, 100, 128, 20, B=2, kv_heads=2, ragged=True)),
    )]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_one(rng):
    op = rng.choice(("rope", "select", "attn", "attn"))
    dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
    d = rng.choice((40, 64, 64, 64, 80, 96, 128, 128))
    kv = rng.choice((1, 2, 4, 5, 8, 10))
    if op == "rope":
        F, H, W = rng.randint(1, 28), _log_int(rng, 8, 72), _log_int(rng, 8, 128)
        # axes as they come; what they leave over of the head is not rotated
        pairs = [rng.randint(0, d // 6), rng.randint(1, d // 6), rng.randint(1, d // 6)]
        pairs[2] += -sum(pairs) % 4
        return _rope(F, H, W, kv * rng.choice((1, 1, 2, 4)), d, pairs, B=rng.choice((1, 2)), kv_heads=kv, dtype=dtype,
                     layout=rng.choice(("interleaved", "halves")), norm=rng.random() < 0.5, origin=rng.choice((0, 0, 17, 1000003)),
                     step=rng.choice((1.0, 1.0, 0.5)), theta=rng.choice((1e4, 256.0)))
    B, group, ragged = rng.choice((1, 2, 2, 4)), rng.choice((1, 1, 1, 4)), rng.random() < 0.4
    N = _log_int(rng, 200, 58000)
    q_block, k_block = rng.choice((32, 64, 100, 128, 128, 256)), rng.choice((64, 64, 128))
    Nk = 0
    if op == "attn" and rng.random() < 0.3:  # few new tokens, each on its own, against a long cache
        N, Nk, q_block, group = rng.choice((1, 1, 3, 8)), _log_int(rng, 300, 200000), 1, rng.choice((1, 4, 8))
    keep = max(1, int(-(-(Nk or N) // k_block) * rng.choice((0.1, 0.125, 0.25, 0.5))))
    return (_select if op == "select" else _attn)(N, kv * group, d, q_block, k_block, keep, B=B, kv_heads=kv, Nk=Nk, dtype=dtype, ragged=ragged)


def _bound(case):
    w = work(case)
    return w["flops"] * (8 if case["dtype"] == "f32" else 1) if case["op"] == "attn" else w["bytes"]


def draw(rng):
    most = {op: max(_bound(c) for c in listed() if c["op"] == op) for op in ("rope", "select", "attn")}
    while True:
        case = _draw_one(rng)
        # the plain form of the attention gathers every run's keys: 2^32 values of them at most
        gathered = work(case)["flops"] / (4 * case["q_block"]) * case["kv_heads"] / case["heads"] if case["op"] == "attn" else 0
        if _bound(case) <= most[case["op"]] and work(case)["bytes"] <= most["rope"] and case["heads"] * case["d"] <= 2048 and gathered <= 1 << 32:
            return case


def _lengths(case):
    """Valid rows of each batch entry of queries and keys: all, or (ragged) a little fewer in every further entry."""
    cut = lambda n: [max(1, n - (n * b) // (2 * case["B"]) - b) if case["ragged"] else n for b in range(case["B"])]  # noqa: E731
    return cut(case["N"]), cut(case["Nk"])


def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    B, heads, kv, d = case["B"], case["heads"], case["kv_heads"], case["d"]
    if case["op"] == "rope":
        n = B * case["F"] * case["H"] * case["W"] * (heads + kv)
        P = case["pf"] + case["ph"] + case["pw"]
        return {"bytes": 2 * n * d * size, "flops": n * (6 * P + (4 * d if case["norm"] else 0))}
    q_len, k_len = _lengths(case)
    runs = [-(-n // case["q_block"]) for n in q_len]
    blocks = [-(-n // case["k_block"]) for n in k_len]
    words = B * kv * -(-case["N"] // case["q_block"]) * -(-case["Nk"] // (32 * case["k_block"])) * 4
    if case["op"] == "select":
        return {"bytes": (sum(q_len) * heads + sum(k_len) * kv) * d * size + words, "flops": 2 * d * kv * sum(r * b for r, b in zip(runs, blocks))}
    keys = [min(case["keep"], b) * case["k_block"] for b in blocks]  # per query
    read = sum(min(n, r * k) for n, r, k in zip(k_len, runs, keys)) * kv
    return {"bytes": (2 * sum(q_len) * heads + 2 * read) * d * size + words, "flops": 4 * d * heads * sum(n * min(k, m) for n, k, m in zip(q_len, keys, k_len))}


# ------------------------------------------------------------------------------------------------ inputs

def _tokens(gen, B, N, heads, d, run, common, dtype):
    """[B,N,heads,d]: N(0,1) noise plus a part shared by `run` neighbours."""
    x = torch.randn(B, N, heads, d, generator=gen, device="cuda")
    if common:
        near = torch.randn(B, -(-N // run), 1, heads, d, generator=gen, device="cuda").expand(-1, -1, run, -1, -1)
        x = (x + common * near.reshape(B, -1, heads, d)[:, :N]) / math.sqrt(1 + common * common)
    return x.to(DTYPE[dtype])


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    B, heads, kv, d, dt = case["B"], case["heads"], case["kv_heads"], case["d"], DTYPE[case["dtype"]]
    if case["op"] == "rope":
        N = case["F"] * case["H"] * case["W"]
        rows = torch.randn(B, N, heads + 2 * kv, d, generator=gen, device="cuda", dtype=torch.float32).to(dt)  # a projection's q | k | v
        gains = (1 + 0.1 * torch.randn(2, d, generator=gen, device="cuda")).to(dt)
        q, k = rows[:, :, :heads], rows[:, :, heads:heads + kv]
        return {"case": case, "q": q, "k": k, "q_gain": gains[0].contiguous(), "k_gain": gains[1].contiguous(),
                "q_out": torch.empty(B, N, heads, d, device="cuda", dtype=dt), "k_out": torch.empty(B, N, kv, d, device="cuda", dtype=dt)}
    N, Nk = case["N"], case["Nk"]
    q = _tokens(gen, B, N, heads, d, 64, 0.5, case["dtype"])
    k = _tokens(gen, B, Nk, kv, d, 64, 0.5, case["dtype"])
    if N == Nk:  # rows of one projection
        v = _tokens(gen, B, Nk, kv, d, 64, 0.0, case["dtype"])
        rows = torch.cat((q, k, v), dim=2)
        q, k, v = rows[:, :, :heads], rows[:, :, heads:heads + kv], rows[:, :, heads + kv:]
    else:
        v = _tokens(gen, B, Nk, kv, d, 64, 0.0, case["dtype"])
    runs, blocks = -(-N // case["q_block"]), -(-Nk // case["k_block"])
    q_len, k_len = _lengths(case)
    state = {"case": case, "q": q, "k": k, "v": v, "q_len": None, "k_len": None}
    if case["ragged"]:
        state["q_len"] = torch.tensor(q_len, dtype=torch.int32, device="cuda")
        state["k_len"] = torch.tensor(k_len, dtype=torch.int32, device="cuda")
    if case["op"] == "select":
        state["blocks"] = torch.zeros(B, kv, runs, -(-blocks // 32), dtype=torch.int32, device="cuda")
        return state
    # the blocks that an earlier selection left: `keep` of those with a key, any of them
    chance = torch.rand(B, kv, runs, blocks, generator=gen, device="cuda")
    has = torch.arange(blocks, device="cuda") * case["k_block"] < torch.tensor(k_len, device="cuda").view(B, 1, 1, 1)
    order = torch.where(has, chance, chance - 2).argsort(dim=-1, descending=True)
    kept = torch.zeros(B, kv, runs, blocks, dtype=torch.bool, device="cuda").scatter_(-1, order[..., :case["keep"]], True) & has
    state["blocks"] = _pack(kept)
    state["out"] = torch.zeros(B, N, heads, d, device="cuda", dtype=dt)
    return state


def _pack(kept):
    """Truth values [.., blocks] as words of 32 bits, block j in bit j % 32 of word j / 32."""
    n = kept.shape[-1]
    bits = torch.nn.functional.pad(kept, (0, -n % 32)).reshape(*kept.shape[:-1], -1, 32).to(torch.int64)
    word = (bits << torch.arange(32, device=kept.device)).sum(dim=-1)
    return torch.where(word >= 1 << 31, word - (1 << 32), word).to(torch.int32)


def _unpack(words, n):
    bits = (words.to(torch.int64).unsqueeze(-1) >> torch.arange(32, device=words.device)) & 1
    return bits.flatten(-2)[..., :n].bool()


# ------------------------------------------------------------------------------------------------ one pass

def run(state):
    op = state["case"]["op"]
    if own:
        return {"rope": _own_rope, "select": _own_select, "attn": _own_attn}[op](state)
    return {"rope": _plain_rope, "select": _plain_select, "attn": _plain_attn}[op](state)


def _own_rope(state):
    import paper_2411_01171_amd as si
    c = state["case"]
    if "rope" not in state:  # the descriptor that a program keeps
        state["rope"] = si.Rope((c["F"], c["H"], c["W"]), (c["pf"], c["ph"], c["pw"]), theta=c["theta"],
                                layout=si.SI_ROPE_HALVES if c["layout"] == "halves" else si.SI_ROPE_INTERLEAVED,
                                origin=(c["origin"], 0, 0), step=(1.0, c["step"], c["step"]), norm_eps=1e-6 if c["norm"] else None,
                                q_gain=state["q_gain"] if c["norm"] else None, k_gain=state["k_gain"] if c["norm"] else None)
    si.si_rope_forward(state["q"], state["k"], state["rope"], state["q_out"], state["k_out"])
    return state["q_out"], state["k_out"]


def _own_select(state):
    import paper_2411_01171_amd as si
    c = state["case"]
    if "workspace" not in state:
        n = si.si_attn_select_workspace_bytes(state["q"], state["k"], c["q_block"], c["k_block"])
        state["workspace"] = torch.empty(n, dtype=torch.uint8, device="cuda")
    si.si_attn_select(state["q"], state["k"], c["q_block"], c["k_block"], c["keep"], state["blocks"], state["workspace"],
                      q_len=state["q_len"], k_len=state["k_len"])
    return state["blocks"]


def _own_attn(state):
    import paper_2411_01171_amd as si
    c = state["case"]
    if "workspace" not in state:
        n = si.si_attn_sparse_workspace_bytes(state["q"], state["k"], c["q_block"], c["k_block"])
        state["workspace"] = torch.empty(n, dtype=torch.uint8, device="cuda")
    si.si_attn_sparse_forward(state["q"], state["k"], state["v"], c["q_block"], c["k_block"], state["blocks"], state["out"],
                              state["workspace"], q_len=state["q_len"], k_len=state["k_len"])
    return state["out"]


def _plain_rope(state):
    c, q, k = state["case"], state["q"], state["k"]
    n = torch.arange(c["F"] * c["H"] * c["W"], device=q.device)
    f, h, w = n // (c["H"] * c["W"]), n // c["W"] % c["H"], n % c["W"]

    def angle(position, pairs):  # positions reach 10^6: 64 bits
        return position.double().unsqueeze(-1) * c["theta"] ** (-torch.arange(pairs, device=q.device, dtype=torch.float64) / max(1, pairs))

    a = torch.cat((angle(f + c["origin"], c["pf"]), angle(h * c["step"], c["ph"]), angle(w * c["step"], c["pw"])), dim=-1)
    cos, sin = a.cos().float().unsqueeze(1), a.sin().float().unsqueeze(1)  # [N, 1, P]
    P = a.shape[-1]

    def turn(x, gain):
        x = x.float()
        if c["norm"]:
            x = x * torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + 1e-6) * gain.float()
        if c["layout"] == "halves":
            x1, x2 = x[..., :P], x[..., P:2 * P]
            y = torch.cat((x1 * cos - x2 * sin, x1 * sin + x2 * cos, x[..., 2 * P:]), dim=-1)
        else:
            x1, x2 = x[..., 0:2 * P:2], x[..., 1:2 * P:2]
            y = torch.cat((torch.stack((x1 * cos - x2 * sin, x1 * sin + x2 * cos), dim=-1).flatten(-2), x[..., 2 * P:]), dim=-1)
        return y.to(q.dtype)

    return turn(q, state["q_gain"]), turn(k, state["k_gain"])


def _rows(case, length, n, device):
    """[B, n] truth values: rows that a batch entry has."""
    at = torch.arange(n, device=device)
    return (at < length.view(-1, 1)) if length is not None else (at < n).expand(case["B"], n)


def _plain_select(state):
    c, q, k = state["case"], state["q"], state["k"]
    B, N, heads, d = q.shape
    Nk, kv = k.shape[1], k.shape[2]
    runs, blocks = -(-N // c["q_block"]), -(-Nk // c["k_block"])
    q_row, k_row = _rows(c, state["q_len"], N, q.device), _rows(c, state["k_len"], Nk, q.device)

    def means(x, row, length, count):  # float64: whether a block is the last one kept can hang on any digit
        x = x.double().masked_fill(~row.view(B, -1, 1, 1), 0.0).flatten(3)
        x = torch.nn.functional.pad(x, (0, 0, 0, 0, 0, count * length - x.shape[1])).view(B, count, length, x.shape[2], -1)
        have = torch.nn.functional.pad(row, (0, count * length - row.shape[1])).reshape(B, count, length).sum(dim=2)
        return x.sum(dim=2), have

    qs, q_have = means(q, q_row, c["q_block"], runs)
    ks, k_have = means(k, k_row, c["k_block"], blocks)
    group = heads // kv
    qm = qs.view(B, runs, kv, group, d).sum(dim=3) / (q_have * group).clamp(min=1).view(B, runs, 1, 1)
    km = ks / k_have.clamp(min=1).view(B, blocks, 1, 1)
    score = torch.matmul(qm.transpose(1, 2).contiguous(), km.permute(0, 2, 3, 1).contiguous())  # [B, kv, runs, blocks]
    score = torch.where(score.isnan(), -math.inf, score)
    has = (k_have > 0).view(B, 1, 1, blocks)
    rank = has.to(torch.float64).expand_as(score)  # blocks without a key come last, whatever their score
    order = torch.where(has, score, -math.inf).argsort(dim=-1, descending=True, stable=True)
    order = order.gather(-1, rank.gather(-1, order).argsort(dim=-1, descending=True, stable=True))
    kept = torch.zeros_like(score, dtype=torch.bool).scatter_(-1, order[..., :c["keep"]], True)
    return _pack(kept & has & (q_have > 0).view(B, 1, runs, 1))


def _plain_attn(state):
    c, q, k, v = state["case"], state["q"], state["k"], state["v"]
    B, N, heads, d = q.shape
    Nk, kv = k.shape[1], k.shape[2]
    qb, kb, group = c["q_block"], c["k_block"], heads // kv
    runs, blocks, most = -(-N // qb), -(-Nk // kb), min(c["keep"], -(-Nk // kb))
    k_row = torch.nn.functional.pad(_rows(c, state["k_len"], Nk, q.device), (0, blocks * kb - Nk))
    kept = _unpack(state["blocks"], blocks)
    kept, at = kept.to(torch.int8).sort(dim=-1, descending=True, stable=True)
    kept, at = kept[..., :most].bool(), at[..., :most]  # [B, kv, runs, most]

    def gather(x):  # [B, kv, runs, most * kb, d] in 32 bits, rows that are not there as zeros
        x = torch.nn.functional.pad(x.transpose(1, 2), (0, 0, 0, blocks * kb - Nk)).reshape(B, kv, blocks, kb * d)
        x = x.gather(2, at.flatten(2).unsqueeze(-1).expand(-1, -1, -1, kb * d))
        return x.view(B, kv, runs, most * kb, d).float().masked_fill(~there.unsqueeze(-1), 0.0)

    there = k_row.reshape(B, 1, blocks, kb).expand(-1, kv, -1, -1).gather(2, at.flatten(2).unsqueeze(-1).expand(-1, -1, -1, kb))
    there = (there.view(B, kv, runs, most, kb) & kept.unsqueeze(-1)).flatten(3)
    rows = torch.nn.functional.pad(q, (0, 0, 0, 0, 0, runs * qb - N)).view(B, runs, qb, kv, group, d)
    rows = rows.permute(0, 3, 1, 2, 4, 5).reshape(B, kv, runs, qb * group, d).float()
    s = torch.matmul(rows, gather(k).transpose(-1, -2)) * (1.0 / math.sqrt(d))
    s = s.masked_fill_(~there.unsqueeze(-2), -math.inf)
    top = s.amax(dim=-1, keepdim=True)
    p = torch.exp(s.sub_(torch.where(top.isinf(), 0.0, top)))
    del s
    total = p.sum(dim=-1, keepdim=True)
    o = torch.matmul(p, gather(v)) / torch.where(total == 0, 1.0, total)
    o = o.view(B, kv, runs, qb, group, d).permute(0, 2, 3, 1, 4, 5).reshape(B, runs * qb, heads, d)[:, :N]
    return o.masked_fill(~_rows(c, state["q_len"], N, q.device).view(B, N, 1, 1), 0.0).to(q.dtype)


# ------------------------------------------------------------------------------------------------ 64 bits

def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "rope":
        return _exact_rope(case, state)
    if case["op"] == "select":
        return None  # whole numbers
    return _exact_attn(case, state)


def _exact_rope(case, state):
    """Every pair of channels as a complex number times e^(i angle), one axis after the other."""
    F, H, W = case["F"], case["H"], case["W"]
    P = case["pf"] + case["ph"] + case["pw"]
    grid = torch.meshgrid(*(torch.arange(n, device="cuda", dtype=torch.float64) for n in (F, H, W)), indexing="ij")
    places = (grid[0] + case["origin"], grid[1] * case["step"], grid[2] * case["step"])
    turns = torch.empty(F, H, W, P, device="cuda", dtype=torch.complex128)
    p = 0
    for place, pairs in zip(places, (case["pf"], case["ph"], case["pw"])):
        for i in range(pairs):
            turns[..., p] = torch.polar(torch.ones_like(place), place * math.pow(case["theta"], -i / pairs))
            p += 1
    turns = turns.view(1, F * H * W, 1, P)
    outs = []
    for x, gain in ((state["q"], state["q_gain"]), (state["k"], state["k_gain"])):
        x = x.double()
        if case["norm"]:
            x = x / (x.pow(2).sum(dim=-1, keepdim=True) / case["d"] + 1e-6).sqrt() * gain.double()
        y = x.clone()
        if case["layout"] == "halves":
            z = torch.complex(x[..., :P].contiguous(), x[..., P:2 * P].contiguous()) * turns
            y[..., :P], y[..., P:2 * P] = z.real, z.imag
        else:
            z = torch.complex(x[..., 0:2 * P:2].contiguous(), x[..., 1:2 * P:2].contiguous()) * turns
            y[..., 0:2 * P:2], y[..., 1:2 * P:2] = z.real, z.imag
        outs.append(y)
    return tuple(outs)


def _exact_attn(case, state):
    """Dense scores of a run of queries and head at a time, the keys of blocks that are not listed left out."""
    if work(case)["flops"] * case["Nk"] / (min(case["keep"] * case["k_block"], case["Nk"])) > 4e13:
        return None  # 64-bit products of every score: too long
    q, k, v = state["q"], state["k"], state["v"]
    out = torch.zeros(q.shape, device="cuda", dtype=torch.float64)
    group, kb = case["heads"] // case["kv_heads"], case["k_block"]
    q_len, k_len = _lengths(case)
    listed_blocks = state["blocks"].cpu().numpy().view("uint32")
    block_of = torch.arange(case["Nk"], device="cuda") // kb
    for b in range(case["B"]):
        for h in range(case["heads"]):
            words = torch.from_numpy(listed_blocks[b, h // group].astype("int64")).to("cuda")  # [runs, words]
            keys, values = k[b, :k_len[b], h // group].double().t().contiguous(), v[b, :k_len[b], h // group].double().contiguous()
            at = block_of[:k_len[b]]
            step = max(1, int(2e8 / k_len[b]))
            for n in range(0, q_len[b], step):
                m = min(q_len[b], n + step)
                run_of = torch.arange(n, m, device="cuda") // case["q_block"]
                first = int(run_of[0])
                inside = ((words[first:int(run_of[-1]) + 1][:, at // 32] >> (at % 32)) & 1).bool()[run_of - first]
                s = (q[b, n:m, h].double() @ keys / math.sqrt(case["d"])).masked_fill(~inside, -math.inf)
                p = torch.softmax(s, dim=-1)
                out[b, n:m, h] = torch.where(inside.any(dim=-1, keepdim=True), p, 0.0) @ values
    return out
