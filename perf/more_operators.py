"""Operators of a cache of keys and values held in 4 bits: storing tokens and reading them back, attention of new tokens over the
cache with the weight that every cached token received, eviction by that weight; sizes, inputs, the plain form, one pass and the
work that it cannot do without.

A case is one call as a program makes it that produces a video frame by frame, or a token at a time: new keys and values lie
interleaved in the rows of one projection, those of earlier frames in the cache.  A head's channels are held in groups of 32:
e2m1 codes (0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign, the even channel in a byte's low half) times 2^(s - 127), one byte s a group.
"""
import math

import torch

own = False  # True: run() calls the library

DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------------------------------------ cases

def _store(N, heads, d, *, B=2, capacity=0, at=0, dtype="bf16", ragged=False):
    return {"op": "store", "B": B, "N": N, "kv_heads": heads, "d": d, "capacity": capacity or at + N, "at": at, "dtype": dtype, "ragged": ragged}


def _attn(N, heads, d, Nk, *, B=2, kv_heads=0, run=0, weights=False, dtype="bf16", ragged=False):
    return {"op": "attn", "B": B, "N": N, "heads": heads, "kv_heads": kv_heads or heads, "d": d, "Nk": Nk, "run": run, "weights": weights,
            "dtype": dtype, "ragged": ragged}


def _evict(Nk, heads, d, keep, *, B=1, first=0, last=0, ragged=False):
    return {"op": "evict", "B": B, "Nk": Nk, "kv_heads": heads, "d": d, "keep": keep, "first": first, "last": last, "ragged": ragged}


def listed():
    return [dict(case, name=name) for name, case in (
        # the new token of four sequences, 8 key heads of 128, at the end of what the cache has: all latency
        ("store_token", _store(1, 8, 128, B=4, capacity=8192, at=8191)),
        # a frame of the largest spatial block (72x128 map, 5 heads of 64), both guidance halves, behind six others
        ("store_frame", _store(9216, 5, 64, capacity=64512, at=55296)),
        # all 25 frames of that level, as a prompt brings them
        ("store_video", _store(230400, 5, 64)),
        # padded batch in single precision, heads of 40
        ("store_f32_padded", _store(4050, 8, 40, B=3, capacity=5000, at=17, dtype="f32", ragged=True)),
        # one token of the deepest level's heads against one 16x16 frame: all latency
        ("attn_16x16", _attn(1, 20, 64, 256, B=1)),
        # one new token against a long cache of frames: 32 query heads share 8 key / value heads
        ("attn_one_token", _attn(1, 32, 128, 115200, B=4, kv_heads=8)),
        # eight tokens at once, each after the other (a guess that is checked), padded batch, weights for the eviction
        ("attn_tokens_weights", _attn(8, 32, 128, 57600, kv_heads=8, run=1, weights=True, ragged=True)),
        # a frame of the second level (32x32 map, 10 heads of 64) over itself and 25 earlier ones, weights for the eviction
        ("attn_32x32_weights", _attn(1024, 10, 64, 26624, weights=True)),
        # a frame of the largest spatial block over itself and six earlier ones: the largest call
        ("attn_72x128", _attn(9216, 5, 64, 64512)),
        # single precision, two frames of 45x45 behind five others, each after the other, heads of 80
        ("attn_f32_frames", _attn(4050, 8, 80, 14175, B=1, run=2025, dtype="f32")),
        # a short cache cut to half: all latency
        ("evict_4096", _evict(4096, 8, 64, 2048, first=4, last=256)),
        # a long one of padded sequences cut to a quarter, the latest frame kept whole
        ("evict_long_padded", _evict(115200, 8, 128, 28800, B=4, first=4, last=1024, ragged=True)),
    )]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_one(rng):
    op = rng.choice(("store", "attn", "attn", "attn", "evict"))
    dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
    d = rng.choice((40, 64, 64, 64, 80, 96, 128, 128))
    B, kv, ragged = rng.choice((1, 2, 2, 3, 4)), rng.choice((1, 2, 4, 5, 8, 10)), rng.random() < 0.4
    if op == "store":
        N, at = _log_int(rng, 1, 230400), rng.choice((0, 0, 1, 1000, 60000))
        return _store(N, kv, d, B=B, capacity=at + N + rng.choice((0, 0, 5)), at=at, dtype=dtype, ragged=ragged)
    if op == "evict":
        Nk = _log_int(rng, 500, 120000)
        keep = max(8, int(Nk * rng.choice((0.05, 0.25, 0.25, 0.5, 0.9))))
        return _evict(Nk, kv, d, keep, B=B, first=rng.choice((0, 0, 4)), last=rng.randint(0, keep // 2 - 4) if keep > 16 else 0, ragged=ragged)
    weights, group = rng.random() < 0.4, rng.choice((1, 1, 2, 4, 8))
    if rng.random() < 0.5:  # new tokens, one or a few
        N, Nk = rng.choice((1, 1, 1, 2, 5, 8, 16)), _log_int(rng, 200, 200000)
        return _attn(N, kv * group, d, max(N, Nk), B=B, kv_heads=kv, run=rng.choice((0, 1)), weights=weights, dtype=dtype, ragged=ragged)
    # one frame, or a few of them one after the other
    frame, frames = _log_int(rng, 100, 9216), rng.choice((1, 1, 1, 2, 3))
    N = frame * frames
    return _attn(N, kv * group, d, N + frame * rng.randint(0, 12), B=B, kv_heads=kv, run=frame if frames > 1 else 0, weights=weights, dtype=dtype, ragged=ragged)


def _bound(case):
    w = work(case)
    return max(w["bytes"] / 5e12, w["flops"] * (12 if case["dtype"] == "f32" else 1) / 1.2e15) if case["op"] == "attn" else w["bytes"]


def draw(rng):
    most = {op: max(_bound(c) for c in listed() if c["op"] == op) for op in ("store", "attn", "evict")}
    while True:
        case = _draw_one(rng)
        # the plain form of the attention keeps every score: 2^32.5 of them at most
        scores = case["B"] * case["heads"] * case["N"] * case["Nk"] if case["op"] == "attn" else 0
        if _bound(case) <= most[case["op"]] and scores <= 6e9 and case.get("heads", 0) * case["d"] <= 4096 and work(case)["bytes"] <= 1.6e9:
            return case


def _lengths(case, n):
    """Tokens that count of each batch entry: all, or (ragged) a little fewer in every further entry."""
    return [max(1, n - (n * b) // (2 * case["B"]) - b) if case["ragged"] else n for b in range(case["B"])]


def work(case):
    B, kv, d = case["B"], case["kv_heads"], case["d"]
    held = 2 * (d // 2 + -(-d // 32))  # bytes of a token's key and value in the cache
    if case["op"] == "evict":
        n = sum(_lengths(case, case["Nk"]))
        kept = sum(min(m, case["keep"]) for m in _lengths(case, case["Nk"]))
        return {"bytes": kv * (4 * n + kept * (2 * held + 8)), "flops": kv * n}
    size = 4 if case["dtype"] == "f32" else 2
    n = sum(_lengths(case, case["N"]))
    if case["op"] == "store":
        return {"bytes": n * kv * (4 * d * size + 2 * held + 4), "flops": 10 * n * kv * d}
    pairs, keys = 0, 0
    for q, k in zip(_lengths(case, case["N"]), _lengths(case, case["Nk"])):
        r = case["run"] or q
        ends = [min(k, max(0, k - q + min(q, e))) for e in range(r, q + r, r)]
        pairs += sum(max(0, min(r, q - i * r)) * e for i, e in enumerate(ends))
        keys += ends[-1]
    return {"bytes": 2 * n * case["heads"] * d * size + kv * keys * (held + (8 if case["weights"] else 0)), "flops": 4 * d * case["heads"] * pairs}


# ------------------------------------------------------------------------------------------------ inputs

def _tokens(gen, B, N, heads, d, common=0.0, run=64):
    """[B,N,heads,d] in 32 bits: N(0,1) noise plus a part shared by `run` neighbours."""
    x = torch.randn(B, N, heads, d, generator=gen, device="cuda")
    if common:
        near = torch.randn(B, -(-N // run), 1, heads, d, generator=gen, device="cuda").expand(-1, -1, run, -1, -1)
        x = (x + common * near.reshape(B, -1, heads, d)[:, :N]) / math.sqrt(1 + common * common)
    return x


def _lens(case, n):
    return torch.tensor(_lengths(case, n), dtype=torch.int32, device="cuda") if case["ragged"] else None


def _sizes(case):
    """Groups of a head, and bytes that a token's scales take."""
    groups = -(-case["d"] // 32)
    return groups, (0, 1, 2, 4, 4)[groups]


def _empty_cache(case, capacity):
    groups, scales = _sizes(case)
    new = lambda n: torch.zeros(case["B"], case["kv_heads"], capacity, n, dtype=torch.uint8, device="cuda")  # noqa: E731
    return {"k_codes": new(16 * groups), "k_scales": new(scales), "v_codes": new(16 * groups), "v_scales": new(scales)}


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    B, kv, d = case["B"], case["kv_heads"], case["d"]
    if case["op"] == "store":
        dt = DTYPE[case["dtype"]]
        k = _tokens(gen, B, case["N"], kv, d, 0.5).to(dt)
        v = _tokens(gen, B, case["N"], kv, d).to(dt)
        rows = torch.cat((k, v), dim=2)  # of one projection
        out = torch.zeros(B, case["N"], 2 * kv, d, device="cuda", dtype=dt)
        return {"case": case, "k": rows[:, :, :kv], "v": rows[:, :, kv:], "k_out": out[:, :, :kv], "v_out": out[:, :, kv:], "length": _lens(case, case["N"]),
                "at": torch.full((B,), case["at"], dtype=torch.int32, device="cuda"), "cache": _empty_cache(case, case["capacity"]),
                "weight": torch.rand(B, kv, case["capacity"], generator=gen, device="cuda")}
    Nk = case["Nk"]
    cache = _empty_cache(case, Nk)
    for b in range(B):
        for name, common in (("k", 0.5), ("v", 0.0)):
            codes, scales = _quantise(_tokens(gen, 1, Nk, kv, d, common)[0].to(torch.bfloat16).float().transpose(0, 1))
            cache[name + "_codes"][b], cache[name + "_scales"][b] = codes, scales
    # what earlier tokens gave: a few cached tokens got most of it, some nothing yet
    weight = (torch.randn(B, kv, Nk, generator=gen, device="cuda") * 1.5 - 1).exp()
    weight = weight.masked_fill(torch.rand(B, kv, Nk, generator=gen, device="cuda") < 0.02, 0.0)
    state = {"case": case, "cache": cache, "weight": weight, "k_len": _lens(case, Nk), "weight_out": torch.zeros_like(weight)}
    if case["op"] == "attn":
        rows = _tokens(gen, B, case["N"], case["heads"] + 2 * kv, d, 0.5).to(DTYPE[case["dtype"]])  # a projection's q | k | v
        q = rows[:, :, :case["heads"]]
        return dict(state, q=q, q_len=_lens(case, case["N"]), out=torch.zeros(q.shape, device="cuda", dtype=q.dtype))
    return dict(state, cut=_empty_cache(case, case["keep"]), weight_out=torch.zeros(B, kv, case["keep"], device="cuda"),
                kept=torch.full((B, kv, case["keep"]), -1, dtype=torch.int32, device="cuda"), cut_len=torch.zeros(B, dtype=torch.int32, device="cuda"))


# ------------------------------------------------------------------------------------------------ one pass

def run(state):
    op = state["case"]["op"]
    if own:
        return {"store": _own_store, "attn": _own_attn, "evict": _own_evict}[op](state)
    return {"store": _plain_store, "attn": _plain_attn, "evict": _plain_evict}[op](state)


def _own_cache(state, name):
    import paper_2411_01171_amd as si
    c = state[name]
    if "k_codes" in c:  # the descriptor that a program keeps
        c["own"] = si.Cache4(c.pop("k_codes"), c.pop("k_scales"), c.pop("v_codes"), c.pop("v_scales"), state["case"]["d"])
    return c["own"]


def _own_store(state):
    import paper_2411_01171_amd as si
    cache = _own_cache(state, "cache")
    si.si_cache4_store(state["k"], state["v"], cache, first=state["at"], length=state["length"], weight=state["weight"])
    si.si_cache4_load(cache, state["k_out"], state["v_out"], first=state["at"], length=state["length"])
    return state["k_out"], state["v_out"], state["weight"]


def _own_attn(state):
    import paper_2411_01171_amd as si
    c, cache = state["case"], _own_cache(state, "cache")
    if "workspace" not in state:
        n = si.si_cache4_attn_workspace_bytes(state["q"], cache, weights=c["weights"])
        state["workspace"] = torch.empty(n, dtype=torch.uint8, device="cuda")
    weights = {"weight_in": state["weight"], "weight_out": state["weight_out"], "decay": 0.99} if c["weights"] else {}
    si.si_cache4_attn_forward(state["q"], cache, state["out"], state["workspace"], q_len=state["q_len"], k_len=state["k_len"], run=c["run"], **weights)
    return (state["out"], state["weight_out"]) if c["weights"] else state["out"]


def _own_evict(state):
    import paper_2411_01171_amd as si
    c, cache, cut = state["case"], _own_cache(state, "cache"), _own_cache(state, "cut")
    if "workspace" not in state:
        state["workspace"] = torch.empty(si.si_cache4_evict_workspace_bytes(cache, c["keep"]), dtype=torch.uint8, device="cuda")
    si.si_cache4_evict(cache, state["weight"], c["keep"], cut, state["weight_out"], state["kept"], state["cut_len"], state["workspace"],
                       first=c["first"], last=c["last"], k_len=state["k_len"])
    return cut.k_codes, cut.k_scales, cut.v_codes, cut.v_scales, state["weight_out"], state["kept"], state["cut_len"]


def _quantise(x):
    """Values [.., d] in 32 bits as codes [.., 16 groups] and scales [.., bytes].  Every step is exact."""
    d = x.shape[-1]
    groups = -(-d // 32)
    x = torch.nn.functional.pad(x, (0, 32 * groups - d)).unflatten(-1, (groups, 32))
    most = x.abs().amax(dim=-1)  # a NaN among them is one
    # the smallest power of two of which the largest magnitude is at most seven times: up from its own binade's where the fraction passes 1.75
    s = (((most.view(torch.int32) + 0x1FFFFF) >> 23) - 2).clamp(2, 252)
    y = x * ((254 - s) << 23).view(torch.float32).unsqueeze(-1)
    a = y.abs()  # to the nearest value, ties to the even code
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5)) | (x.signbit().to(torch.uint8) << 3)
    fine = most.isfinite()
    s = torch.where(fine, s, 255)
    code = torch.where(fine.unsqueeze(-1), code, 0).flatten(-2)
    return code[..., 0::2] | (code[..., 1::2] << 4), torch.nn.functional.pad(s, (0, (0, 1, 2, 4, 4)[groups] - groups)).to(torch.uint8)


def _values(codes, scales, d):
    """What codes and scales stand for, [.., d] in 32 bits."""
    groups = -(-d // 32)
    grid = torch.tensor((0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0), device=codes.device)
    grid = torch.cat((grid, -grid))
    code = torch.stack((codes & 15, codes >> 4), dim=-1).flatten(-2).to(torch.int32)
    s = scales[..., :groups].to(torch.int32)
    power = torch.where(s == 255, math.nan, (s << 23).view(torch.float32))
    return (grid[code].unflatten(-1, (groups, 32)) * power.unsqueeze(-1)).flatten(-2)[..., :d]


def _plain_store(state):
    c, cache = state["case"], state["cache"]
    B, N, at = c["B"], c["N"], c["at"]
    there = torch.arange(N, device="cuda").view(1, 1, N, 1) < (N if state["length"] is None else state["length"].view(B, 1, 1, 1))
    for name in ("k", "v"):
        codes, scales = _quantise(state[name].float().transpose(1, 2))
        new_codes, new_scales = (cache[name + part][:, :, at:at + N] for part in ("_codes", "_scales"))
        new_codes.copy_(torch.where(there, codes, new_codes))
        new_scales.copy_(torch.where(there, scales, new_scales))
        out = state[name + "_out"]
        out.copy_(torch.where(there.transpose(1, 2), _values(new_codes, new_scales, c["d"]).transpose(1, 2).to(out.dtype), out))
    state["weight"][:, :, at:at + N].masked_fill_(there.squeeze(-1), 0.0)
    return state["k_out"], state["v_out"], state["weight"]


def _seen(case, q_len, k_len):
    """[B, N, 1]: keys that a query sees, the first so many; 0 behind the queries that count."""
    q = torch.tensor(_lengths(case, case["N"]), device="cuda") if q_len is None else q_len
    k = torch.tensor(_lengths(case, case["Nk"]), device="cuda") if k_len is None else k_len
    q, k, n = q.view(-1, 1).long(), k.view(-1, 1).long(), torch.arange(case["N"], device="cuda")
    end = torch.minimum((n // case["run"] + 1) * case["run"], q) if case["run"] else q
    return torch.where(n < q, (k - q + end).clamp(min=0), 0).unsqueeze(-1)


def _plain_attn(state):
    c, q = state["case"], state["q"]
    B, N, heads, d = q.shape
    kv, Nk = c["kv_heads"], c["Nk"]
    group = heads // kv
    k, v = (_values(state["cache"][n + "_codes"], state["cache"][n + "_scales"], d) for n in ("k", "v"))  # [B, kv, Nk, d]
    seen = _seen(c, state["q_len"], state["k_len"])
    hidden = (torch.arange(Nk, device="cuda") >= seen).view(B, 1, N, 1, Nk)
    rows = q.float().view(B, N, kv, group, d).transpose(1, 2).reshape(B, kv, N * group, d)
    s = torch.matmul(rows, k.transpose(-1, -2).contiguous()).mul_(1.0 / math.sqrt(d))
    s.view(B, kv, N, group, Nk).masked_fill_(hidden, -math.inf)
    top = s.amax(dim=-1, keepdim=True)
    p = s.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = p.sum(dim=-1, keepdim=True)
    p.div_(torch.where(total == 0, 1.0, total))
    o = torch.matmul(p, v).view(B, kv, N, group, d).transpose(1, 2).reshape(B, N, heads, d).to(q.dtype)
    if not c["weights"]:
        return o
    j = torch.arange(Nk, device="cuda")
    counts = (j < Nk if state["k_len"] is None else j < state["k_len"].view(B, 1)).view(-1, 1, Nk)
    return o, torch.where(counts, state["weight"] * 0.99 + p.sum(dim=-2), 0.0)


def _plain_evict(state):
    c, cache = state["case"], state["cache"]
    B, kv, Nk, keep = c["B"], c["kv_heads"], c["Nk"], c["keep"]
    j = torch.arange(Nk, device="cuda").view(1, 1, Nk)
    length = torch.full((B, 1, 1), Nk, device="cuda") if state["k_len"] is None else state["k_len"].view(B, 1, 1).long()
    w = torch.where(state["weight"].isnan(), -math.inf, state["weight"])
    rank = torch.where(j >= length, 0, torch.where((j < c["first"]) | (j >= length - c["last"]), 2, 1)).expand(B, kv, Nk)
    order = w.argsort(dim=-1, descending=True, stable=True)
    order = order.gather(-1, rank.gather(-1, order).argsort(dim=-1, descending=True, stable=True))[..., :keep]
    n = length.clamp(max=keep)
    there = torch.arange(order.shape[-1], device="cuda").view(1, 1, -1) < n
    at = torch.where(there, order, Nk).sort(dim=-1).values
    at = torch.nn.functional.pad(at, (0, keep - at.shape[-1]), value=Nk)
    there = at < Nk

    def take(x):  # rows that no token is left for stay zero
        x = x.gather(2, at.clamp(max=Nk - 1).unsqueeze(-1).expand(-1, -1, -1, x.shape[-1]))
        return x.masked_fill(~there.unsqueeze(-1), 0)

    parts = [take(cache[p]) for p in ("k_codes", "k_scales", "v_codes", "v_scales")]
    return (*parts, take(state["weight"].unsqueeze(-1)).squeeze(-1), torch.where(there, at, -1).to(torch.int32), n.view(B).to(torch.int32))


# ------------------------------------------------------------------------------------------------ 64 bits

def exact(case, seed):
    if case["op"] == "evict":
        return None  # copies and whole numbers
    return _exact_store(case, prepare(case, seed)) if case["op"] == "store" else _exact_attn(case, prepare(case, seed))


def _exact_store(case, state):
    """Nearest multiple of each value's own step: half a unit below one, then half of its power of two."""
    outs = []
    for x in (state["k"], state["v"]):
        y = torch.zeros(x.shape, device="cuda", dtype=torch.float64)
        for b, n in enumerate(_lengths(case, case["N"])):
            for g in range(0, case["d"], 32):
                part = x[b, :n, :, g:g + 32].double()
                most = part.abs().amax(dim=-1, keepdim=True)
                scale = torch.exp2(torch.ceil(torch.log2(most / 7)).clamp(-125, 125))
                t = part / scale
                step = torch.exp2(torch.floor(torch.log2(t.abs().clamp(min=1.0))) - 1)
                y[b, :n, :, g:g + 32] = (torch.round(t / step) * step).clamp(-6, 6) * scale
        outs.append(y)
    weight = state["weight"].double()
    for b, n in enumerate(_lengths(case, case["N"])):
        weight[b, :, case["at"]:case["at"] + n] = 0
    return outs[0], outs[1], weight


def _unpacked(codes, scales, d):
    """Rows [n, d] in 64 bits: sign, power of two and half of a code, by its bits."""
    code = torch.stack((codes & 15, codes >> 4), dim=-1).flatten(-2).long()[:, :d]
    high, half = (code >> 1) & 3, (code & 1).double()
    size = torch.where(high == 0, half * 0.5, (1 + half * 0.5) * torch.exp2((high - 1).double()))
    power = torch.exp2(scales.double() - 127)[:, torch.arange(d, device=codes.device) // 32]
    return torch.where(code >= 8, -size, size) * power


def _exact_attn(case, state):
    """A head and some rows at a time, over the keys that they see."""
    if work(case)["flops"] > 4e13:
        return None
    q, cache, group = state["q"], state["cache"], case["heads"] // case["kv_heads"]
    out = torch.zeros(q.shape, device="cuda", dtype=torch.float64)
    weight = torch.zeros(state["weight"].shape, device="cuda", dtype=torch.float64)
    for b, (nq, nk) in enumerate(zip(_lengths(case, case["N"]), _lengths(case, case["Nk"]))):
        weight[b, :, :nk] = state["weight"][b, :, :nk].double() * 0.99
        for hk in range(case["kv_heads"]):
            keys, values = (_unpacked(cache[x + "_codes"][b, hk, :nk], cache[x + "_scales"][b, hk, :nk], case["d"]) for x in "kv")
            keys = keys.t().contiguous()
            step = max(1, min(int(2e8 / nk), case["run"] or nq))
            for n in range(0, nq, step):
                m = min(nq, n + step) if not case["run"] else min(nq, n + step, (n // case["run"] + 1) * case["run"])
                end = nk if not case["run"] else max(0, nk - nq + min(nq, (n // case["run"] + 1) * case["run"]))
                if end == 0:
                    continue
                for h in range(hk * group, hk * group + group):
                    p = torch.softmax(q[b, n:m, h].double() @ keys[:, :end] / math.sqrt(case["d"]), dim=-1)
                    out[b, n:m, h] = p @ values[:end]
                    weight[b, hk, :end] += p.sum(dim=0)
    return (out, weight) if case["weights"] else out
