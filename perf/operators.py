"""Timed work of the operators that stand between a decoder's linear layers, one pass per case, through the public calls of the package.

Kinds of work (`case["kind"]`):

* ``attention``  one new token per request against a paged key-value cache: `dps_paged_attention`.
* ``qk``         norms of queries and keys for each head, position rotation, and the write of keys and values into the cache, from the
                 output of the QKV linear: `dps_qk_norm_rope`.
* ``tables``     the block tables, lengths, positions and cache slots of a step, from the request lengths: `dps_extend_block_tables`.
* ``route``      the experts of each token and their weights, from the router's logits: `dps_route_experts`.

A plain form computes in 32 bits (in 64 where a choice falls next to a border) with elementary operations and rounds once at the end.
Lengths follow from the case alone; values, the order of the cache's blocks and everything else follow from the seed.
"""
import math
import random

import numpy as np
import torch

own = False

TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}
# the largest of each kind: bytes of keys and values, tokens x heads x head size, tokens, logits
MOST = {"attention": 2.2e9, "qk": 8192 * 80 * 128, "tables": 65536, "route": 16384 * 256}
FAR = 131072        # positions that the rotation table covers


def listed():
    return [
        # one user's first words on a 4096-wide layer: the smallest call
        {"name": "attention_one_short", "kind": "attention", "requests": 1, "longest": 17, "spread": "same", "heads": 32, "kv_heads": 32, "dim": 128,
         "page": 16, "type": "fp16"},
        # a small batch on a layer of hidden size 8192 (64 query heads, 8 shared key-value heads), medium contexts
        {"name": "attention_8_medium", "kind": "attention", "requests": 8, "longest": 4096, "spread": "even", "heads": 64, "kv_heads": 8, "dim": 128,
         "page": 16, "type": "fp16"},
        # every head with keys of its own, short and long requests mixed, one row of the batch empty
        {"name": "attention_32_mixed", "kind": "attention", "requests": 32, "longest": 3001, "spread": "wide", "heads": 32, "kv_heads": 32, "dim": 128,
         "page": 32, "type": "bf16"},
        # one very long context: the split over its length
        {"name": "attention_one_long", "kind": "attention", "requests": 1, "longest": 131071, "spread": "same", "heads": 64, "kv_heads": 8, "dim": 128,
         "page": 64, "type": "fp16"},
        # a full server; head and page sizes that are no powers of two (the largest work)
        {"name": "attention_112_ragged", "kind": "attention", "requests": 112, "longest": 8190, "spread": "even", "heads": 60, "kv_heads": 10, "dim": 96,
         "page": 24, "type": "bf16"},
        # one decoded token, norms and rotation
        {"name": "qk_one_token", "kind": "qk", "tokens": 1, "heads": 32, "kv_heads": 32, "dim": 128, "rotated": 128, "interleaved": False, "norm": True,
         "page": 16, "padding": 0, "type": "fp16"},
        # half of each head rotated, in neighbouring pairs, a prompt of an odd length padded for a captured graph
        {"name": "qk_999_partial", "kind": "qk", "tokens": 999, "heads": 24, "kv_heads": 6, "dim": 96, "rotated": 48, "interleaved": True, "norm": True,
         "page": 24, "padding": 25, "type": "bf16"},
        # a long prompt on the layer of hidden size 8192
        {"name": "qk_8192_prompt", "kind": "qk", "tokens": 8192, "heads": 64, "kv_heads": 8, "dim": 128, "rotated": 128, "interleaved": False, "norm": True,
         "page": 16, "padding": 0, "type": "fp16"},
        # a decode step of a small batch, padded to the size that its graph was captured for
        {"name": "tables_decode_13", "kind": "tables", "requests": 13, "longest": 4096, "new": "one", "tokens": 16, "page": 16},
        # a mixed step of a large server: long prompts next to decoding requests
        {"name": "tables_mixed_1500", "kind": "tables", "requests": 1500, "longest": 8192, "new": "mixed", "tokens": 65536, "page": 16},
        # eight experts, two of them for each token of a small decode batch
        {"name": "route_8_of_8", "kind": "route", "tokens": 8, "experts": 8, "top": 2, "scoring": "softmax", "groups": 1, "top_groups": 1, "bias": False,
         "scale": 1.0, "type": "fp16"},
        # many experts in groups, sigmoid scores with a bias for balance, a long prompt
        {"name": "route_16384_grouped", "kind": "route", "tokens": 16384, "experts": 256, "top": 8, "scoring": "sigmoid", "groups": 8, "top_groups": 4,
         "bias": True, "scale": 2.5, "type": "bf16"},
    ]


def spread(rng, low, high):
    """A whole number between the two, even over its logarithm."""
    return max(low, min(high, round(math.exp(rng.uniform(math.log(low), math.log(high))))))


def draw(rng):
    kind = rng.choice(["attention", "attention", "qk", "tables", "route"])
    if kind == "tables":
        c = {"kind": kind, "requests": spread(rng, 1, 2000), "longest": spread(rng, 16, 16384), "new": rng.choice(["one", "mixed"]),
             "page": rng.choice([1, 8, 16, 24, 32, 64, 128])}
        return {**c, "tokens": max(c["requests"], spread(rng, c["requests"], MOST[kind]) if c["new"] == "mixed" else c["requests"] + rng.randrange(8))}
    if kind == "route":
        groups = rng.choice([1, 1, 2, 4, 8])
        experts = groups * spread(rng, 4, 512 // groups)
        top_groups = rng.randint(1, groups)
        top = rng.randint(1, min(16, top_groups * (experts // groups)))
        return {"kind": kind, "tokens": spread(rng, 1, MOST[kind] // max(256, experts)), "experts": experts, "top": top,
                "scoring": rng.choice(["softmax", "sigmoid"]), "groups": groups, "top_groups": top_groups, "bias": rng.random() < 0.5,
                "scale": rng.choice([1.0, 2.5]), "type": rng.choice(["fp16", "bf16", "fp32"])}
    kv_heads = rng.choice([1, 2, 4, 5, 8, 16, 32])
    shared = rng.choice([1, 2, 3, 4, 6, 8, 12, 16]) if kv_heads <= 8 else rng.choice([1, 2, 3])
    c = {"kind": kind, "heads": kv_heads * shared, "kv_heads": kv_heads, "dim": rng.choice([64, 80, 96, 128, 128, 128, 192, 256]),
         "page": rng.choice([8, 16, 16, 24, 32, 64, 128]), "type": rng.choice(["fp16", "bf16"])}
    if kind == "qk":
        rotated = rng.choice([c["dim"], c["dim"] // 32 * 16])
        most = min(8192, MOST[kind] // ((c["heads"] + 2 * kv_heads) * c["dim"]))
        return {**c, "tokens": spread(rng, 1, most), "rotated": rotated, "interleaved": rng.random() < 0.5, "norm": rng.random() < 0.75,
                "padding": rng.choice([0, 0, 3])}
    each = 4 * kv_heads * c["dim"]                          # bytes of keys and values of one token
    most = MOST[kind] / each                                # tokens in all
    requests = spread(rng, 1, min(256, int(most // 64)))
    return {**c, "requests": requests, "longest": spread(rng, 1, int(min(131072, most // requests))), "spread": rng.choice(["same", "even", "wide"])}


# ---- what a case holds ------------------------------------------------------------------------------------------------------------
def lengths_of(case):
    """Tokens of each request: all the same, even between nothing and the longest, or mostly short ones."""
    rng, n, longest = random.Random(case["requests"] * 1000003 + case["longest"]), case["requests"], case["longest"]
    if case.get("spread", "even") == "same":
        return [longest] * n
    if case.get("spread") == "wide":
        got = [spread(rng, 1, longest) for _ in range(n)]
    else:
        got = [rng.randint(1, longest) for _ in range(n)]
    got[rng.randrange(n)] = longest
    if n > 4:                                               # a row of the batch that nobody uses
        got[n // 2] = 0
    return got


def new_of(case):
    """Tokens that each request adds in this step."""
    n = case["requests"]
    if case["new"] == "one":
        return [1] * n
    rng = random.Random(case["tokens"] * 31 + n)
    weight = [rng.random() ** 8 for _ in range(n)]          # a few prompts, many single tokens
    room = case["tokens"] - n
    return [1 + int(room * w / sum(weight)) for w in weight]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    kind, dev = case["kind"], "cuda"
    if kind == "route":
        logits = torch.randn((case["tokens"], case["experts"]), generator=g, device=dev).to(TYPES[case["type"]])
        bias = 0.1 * torch.randn((case["experts"],), generator=g, device=dev) if case["bias"] else None
        rows = case["tokens"] * case["top"]                 # what the grouped linears read, kept from step to step
        return {"case": case, "logits": logits, "bias": bias, "token_of_row": torch.empty(rows, dtype=torch.int32, device=dev),
                "expert_of_row": torch.empty(rows, dtype=torch.int32, device=dev), "weights": torch.empty((case["tokens"], case["top"]), device=dev)}
    if kind == "tables":
        page, lengths, new = case["page"], lengths_of(case), new_of(case)
        have = [-(-n // page) for n in lengths]
        need = [-(-(n + m) // page) for n, m in zip(lengths, new)]
        blocks = sum(need) + 7
        order = torch.randperm(blocks, generator=g, device=dev).to(torch.int32)
        width = max(need) + 3
        h = torch.tensor(have, device=dev)
        at = torch.arange(width, device=dev)[None, :]
        first = (torch.cumsum(h, 0) - h)[:, None]
        table = torch.where(at < h[:, None], order[(first + at).clamp(max=blocks - 1)], -1).to(torch.int32)
        granted = order[sum(have):sum(need) + 5]            # a few more than this step takes
        tokens, n = case["tokens"], case["requests"]
        out = {"lengths": torch.empty(n, dtype=torch.int32, device=dev), "starts": torch.empty(n + 1, dtype=torch.int32, device=dev),
               "positions": torch.empty(tokens, dtype=torch.int32, device=dev), "slots": torch.empty(tokens, dtype=torch.int64, device=dev),
               "used": torch.empty(1, dtype=torch.int32, device=dev)}
        return {"case": case, "lengths": torch.tensor(lengths, dtype=torch.int32, device=dev), "new": torch.tensor(new, dtype=torch.int32, device=dev),
                "table": table, "granted": granted, "blocks": blocks, "out": out}
    kv_heads, dim, page, dtype = case["kv_heads"], case["dim"], case["page"], TYPES[case["type"]]
    if kind == "qk":
        tokens, padding = case["tokens"], case["padding"]
        blocks = -(-tokens * 5 // (4 * page)) + 1
        cache = torch.zeros((2, blocks, page, kv_heads, dim), dtype=dtype, device=dev)
        width = (case["heads"] + 2 * kv_heads) * dim
        qkv = torch.randn((tokens + padding, width), generator=g, device=dev).to(dtype)
        slots = torch.randperm(blocks * page, generator=g, device=dev)[:tokens + padding]
        slots[tokens:] = -1                                 # rows that only fill the batch up
        positions = torch.randint(0, FAR, (tokens + padding,), generator=g, device=dev, dtype=torch.int32)
        half = case["rotated"] // 2
        angle = torch.arange(FAR, device=dev, dtype=torch.float64)[:, None] * 500000.0 ** (-torch.arange(half, device=dev, dtype=torch.float64) / half)
        cos_sin = torch.cat([angle.cos(), angle.sin()], 1).float()
        weights = [(1 + 0.2 * torch.randn((dim,), generator=g, device=dev)).to(dtype) for _ in range(2)] if case["norm"] else [None, None]
        return {"case": case, "qkv": qkv, "k_cache": cache[0], "v_cache": cache[1], "slots": slots, "positions": positions, "cos_sin": cos_sin,
                "q_weight": weights[0], "k_weight": weights[1], "eps": 1e-6,
                "q": torch.zeros((tokens + padding, case["heads"], dim), dtype=dtype, device=dev)}
    lengths = lengths_of(case)
    have = [-(-n // page) for n in lengths]
    blocks, width = sum(have) + 3, max(have) + 2
    order = torch.randperm(blocks, generator=g, device=dev).to(torch.int32)
    h = torch.tensor(have, device=dev)
    at = torch.arange(width, device=dev)[None, :]
    first = (torch.cumsum(h, 0) - h)[:, None]
    table = torch.where(at < h[:, None], order[(first + at).clamp(max=blocks - 1)], -1).to(torch.int32)
    cache = torch.empty((2, blocks, page, kv_heads, dim), dtype=dtype, device=dev).normal_(generator=g)
    q = torch.randn((case["requests"], case["heads"], dim), generator=g, device=dev).to(dtype)
    state = {"case": case, "q": q, "k_cache": cache[0], "v_cache": cache[1], "table": table, "lengths": torch.tensor(lengths, dtype=torch.int32, device=dev),
             "longest": max(lengths), "out": torch.empty_like(q)}
    if own:                                                 # the scratch that a serving loop keeps beside its cache
        import paper_2609_34380_b200 as dps
        state["workspace"] = dps.dps_paged_attention_workspace(case["heads"], kv_heads, dim)
    return state


# ---- one pass ---------------------------------------------------------------------------------------------------------------------
def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"attention": attention_own, "qk": qk_own, "tables": tables_own, "route": route_own}[kind](state)
    return {"attention": attention_plain, "qk": qk_plain, "tables": tables_plain, "route": route_plain}[kind](state)


def attention_own(s):
    import paper_2609_34380_b200 as dps
    return dps.dps_paged_attention(s["q"], s["k_cache"], s["v_cache"], s["table"], s["lengths"], out=s["out"], workspace=s["workspace"])


def qk_own(s):
    import paper_2609_34380_b200 as dps
    c = s["case"]
    q = dps.dps_qk_norm_rope(s["qkv"], s["k_cache"], s["v_cache"], s["slots"], s["positions"], s["cos_sin"], s["q_weight"], s["k_weight"],
                             eps=s["eps"], interleaved=c["interleaved"], q_out=s["q"])
    return {"q": q, "k": s["k_cache"], "v": s["v_cache"]}


def tables_own(s):
    import paper_2609_34380_b200 as dps
    o = s["out"]
    dps.dps_extend_block_tables(s["lengths"], s["new"], s["granted"], s["table"], s["case"]["page"], s["blocks"], o["lengths"], o["starts"],
                                o["positions"], o["slots"], o["used"])
    return {**o, "table": s["table"]}


def route_own(s):
    import paper_2609_34380_b200 as dps
    c = s["case"]
    token, expert, weights = dps.dps_route_experts(
        s["logits"], c["top"], s["bias"], dps.DPS_SCORE_SIGMOID if c["scoring"] == "sigmoid" else dps.DPS_SCORE_SOFTMAX, c["groups"], c["top_groups"],
        scale=c["scale"], token_of_row=s["token_of_row"], expert_of_row=s["expert_of_row"], weights=s["weights"])
    return {"token": token, "expert": expert, "weights": weights}


def attention_plain(s):
    c = s["case"]
    q, kv_heads, dim, page = s["q"].float(), c["kv_heads"], c["dim"], c["page"]
    n, pages = q.shape[0], -(-s["longest"] // page)
    at = s["table"][:, :pages].clamp(min=0).long()
    seen = torch.arange(pages * page, device=q.device) < s["lengths"][:, None]                          # [requests][tokens]
    k = s["k_cache"][at].reshape(n, pages * page, kv_heads, dim).float()
    scores = torch.einsum("nghd,nthd->nhgt", q.view(n, kv_heads, -1, dim).transpose(1, 2), k) * dim ** -0.5
    del k
    scores = torch.where(seen[:, None, None, :], scores, -math.inf)
    top = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    v = s["v_cache"][at].reshape(n, pages * page, kv_heads, dim).float()
    out = torch.einsum("nhgt,nthd->nhgd", p, v) / torch.where(total == 0, 1.0, total)
    return out.reshape(n, c["heads"], dim).to(s["q"].dtype)


def rotate_plain(x, cos, sin, rotated, interleaved):
    if not rotated:
        return x
    a, b = (x[..., 0:rotated:2], x[..., 1:rotated:2]) if interleaved else (x[..., :rotated // 2], x[..., rotated // 2:rotated])
    u, v = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([u, v], -1).flatten(-2) if interleaved else torch.cat([u, v], -1)
    return torch.cat([turned, x[..., rotated:]], -1)


def qk_plain(s):
    c = s["case"]
    heads, kv_heads, dim, dtype = c["heads"], c["kv_heads"], c["dim"], s["qkv"].dtype
    x = s["qkv"].view(-1, heads + 2 * kv_heads, dim)
    q, k, v = x[:, :heads].float(), x[:, heads:heads + kv_heads].float(), x[:, heads + kv_heads:]
    if c["norm"]:
        q = q * torch.rsqrt(q.square().mean(-1, keepdim=True) + s["eps"]) * s["q_weight"].float()
        k = k * torch.rsqrt(k.square().mean(-1, keepdim=True) + s["eps"]) * s["k_weight"].float()
    row = s["cos_sin"][s["positions"].long()][:, None, :]
    cos, sin = row[..., :c["rotated"] // 2], row[..., c["rotated"] // 2:]
    q, k = (rotate_plain(t, cos, sin, c["rotated"], c["interleaved"]).to(dtype) for t in (q, k))
    live = s["slots"] >= 0
    s["q"][live] = q[live]
    at = s["slots"][live]
    s["k_cache"].view(-1, kv_heads, dim)[at] = k[live]
    s["v_cache"].view(-1, kv_heads, dim)[at] = v[live]
    return {"q": s["q"], "k": s["k_cache"], "v": s["v_cache"]}


def tables_plain(s):
    c, table, lengths, new, granted = s["case"], s["table"], s["lengths"].long(), s["new"].long(), s["granted"]
    page, tokens = c["page"], c["tokens"]
    have, need = (lengths + page - 1) // page, (lengths + new + page - 1) // page
    taken = torch.cumsum(need - have, 0)                                                                # blocks, this request's with them
    at = torch.arange(table.shape[1], device=table.device)[None, :]
    fresh = (at >= have[:, None]) & (at < need[:, None])
    source = (taken - need)[:, None] + at                                                               # where a fresh block comes from
    table.copy_(torch.where(fresh, granted[source.clamp(0, granted.numel() - 1)], table))
    ends = torch.cumsum(new, 0)
    t = torch.arange(tokens, device=table.device)
    of = torch.searchsorted(ends, t, right=True)
    live = of < lengths.numel()
    of = of.clamp(max=lengths.numel() - 1)
    position = torch.where(live, lengths[of] + t - (ends - new)[of], 0)
    block = table[of, torch.where(live, position // page, 0)].long()
    return {"lengths": (lengths + new).int(), "starts": torch.cat([torch.zeros_like(ends[:1]), ends]).int(), "positions": position.int(),
            "slots": torch.where(live, block * page + position % page, -1), "used": taken[-1:].int(), "table": table}


def route_plain(s):
    c, x = s["case"], s["logits"].double()                  # in 64 bits: two choices may be next to each other
    n, experts = x.shape
    if c["scoring"] == "sigmoid":
        score = 1 / (1 + torch.exp(-x))
    else:
        e = torch.exp(x - x.amax(1, keepdim=True))
        score = e / e.sum(1, keepdim=True)
    choice = score + s["bias"].double() if c["bias"] else score
    if c["groups"] > 1:
        grouped = choice.view(n, c["groups"], -1)
        worth = torch.sort(grouped, dim=2, descending=True)[0][..., :2].sum(2)
        best = torch.sort(worth, dim=1, descending=True, stable=True)[1][:, :c["top_groups"]]
        open_ = torch.zeros_like(worth, dtype=torch.bool).scatter_(1, best, True)
        choice = torch.where(open_[:, :, None], grouped, -math.inf).view(n, experts)
    expert = torch.sort(choice, dim=1, descending=True, stable=True)[1][:, :c["top"]]
    weights = torch.gather(score, 1, expert)
    weights = weights / weights.sum(1, keepdim=True) * c["scale"]
    token = torch.arange(n, device=x.device)[:, None].expand(-1, c["top"])
    return {"token": token.reshape(-1).int(), "expert": expert.reshape(-1).int(), "weights": weights.float()}


# ---- what it cannot do without ----------------------------------------------------------------------------------------------------
def work(case):
    kind = case["kind"]
    if kind == "attention":
        total, n = sum(lengths_of(case)), case["requests"]
        pages = sum(-(-x // case["page"]) for x in lengths_of(case))
        return {"bytes": 4 * total * case["kv_heads"] * case["dim"] + 4 * n * case["heads"] * case["dim"] + 4 * pages + 4 * n,
                "flops": 4 * total * case["heads"] * case["dim"]}
    if kind == "qk":
        n, values = case["tokens"], (case["heads"] + 2 * case["kv_heads"]) * case["dim"]
        return {"bytes": n * (4 * values + 4 * case["rotated"] + 12) + 8 * case["padding"] + (4 * case["dim"] if case["norm"] else 0),
                "flops": n * (case["heads"] + case["kv_heads"]) * ((4 * case["dim"] if case["norm"] else 0) + 3 * case["rotated"])}
    if kind == "tables":
        n, tokens = case["requests"], case["tokens"]
        fresh = sum(-(-(a + b) // case["page"]) - -(-a // case["page"]) for a, b in zip(lengths_of(case), new_of(case)))
        return {"bytes": 16 * n + 12 * tokens + 8 * fresh + 4 * n, "flops": 4 * tokens}
    size = {"fp16": 2, "bf16": 2, "fp32": 4}[case["type"]]
    return {"bytes": case["tokens"] * (case["experts"] * size + 12 * case["top"]) + (4 * case["experts"] if case["bias"] else 0),
            "flops": 8 * case["tokens"] * case["experts"]}


# ---- the definition, in 64 bits ---------------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"attention": attention_exact, "qk": qk_exact, "tables": tables_exact, "route": route_exact}[case["kind"]](case, s)


def attention_exact(case, s):
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    page, share = case["page"], case["heads"] // case["kv_heads"]
    for i, n in enumerate(lengths_of(case)):
        if n == 0:
            continue
        blocks = s["table"][i, :-(-n // page)].long()
        keys = s["k_cache"].index_select(0, blocks).flatten(0, 1)[:n].double().permute(1, 0, 2)       # [kv heads][tokens][dim]
        values = s["v_cache"].index_select(0, blocks).flatten(0, 1)[:n].double().permute(1, 0, 2)
        query = s["q"][i].double().reshape(case["kv_heads"], share, case["dim"])
        logit = torch.bmm(query, keys.transpose(1, 2)) / math.sqrt(case["dim"])
        out[i] = torch.bmm(torch.softmax(logit, 2), values).reshape(case["heads"], case["dim"])
    return out


def qk_exact(case, s):
    heads, kv_heads, dim, n, half = case["heads"], case["kv_heads"], case["dim"], case["tokens"], case["rotated"] // 2
    x = s["qkv"][:n].double().reshape(n, heads + 2 * kv_heads, dim)
    turn = torch.view_as_complex(s["cos_sin"].double()[s["positions"][:n].long()].reshape(n, 1, 2, half).transpose(2, 3).contiguous())

    def one(part, weight):
        if weight is not None:
            part = part / (part.pow(2).sum(2, keepdim=True) / dim + s["eps"]).sqrt() * weight.double()
        part = part.clone()
        if case["interleaved"]:
            z = turn * torch.view_as_complex(part[..., :2 * half].reshape(n, -1, half, 2))
            part[..., :2 * half] = torch.view_as_real(z).reshape(n, -1, 2 * half)
        else:
            z = turn * torch.complex(part[..., :half], part[..., half:2 * half])
            part[..., :half], part[..., half:2 * half] = z.real, z.imag
        return part
    q = s["q"].double()
    q[:n] = one(x[:, :heads], s["q_weight"])
    k, v = s["k_cache"].double(), s["v_cache"].double()
    k.view(-1, kv_heads, dim).index_copy_(0, s["slots"][:n], one(x[:, heads:heads + kv_heads], s["k_weight"]))
    v.view(-1, kv_heads, dim).index_copy_(0, s["slots"][:n], x[:, heads + kv_heads:])
    return {"q": q, "k": k, "v": v}


def tables_exact(case, s):
    page, table, granted = case["page"], s["table"].cpu().numpy().copy(), s["granted"].cpu().numpy()
    positions, slots = np.zeros(case["tokens"], np.int32), np.full(case["tokens"], -1, np.int64)
    lengths, starts, taken, t = [], [0], 0, 0
    for i, (n, m) in enumerate(zip(lengths_of(case), new_of(case))):
        for j in range(-(-n // page), -(-(n + m) // page)):
            table[i, j] = granted[taken]
            taken += 1
        p = np.arange(n, n + m)
        positions[t:t + m], slots[t:t + m] = p, table[i, p // page].astype(np.int64) * page + p % page
        t += m
        lengths.append(n + m)
        starts.append(t)
    return {"lengths": np.array(lengths, np.int32), "starts": np.array(starts, np.int32), "positions": positions, "slots": slots,
            "used": np.array([taken], np.int32), "table": table}


def route_exact(case, s):
    x = s["logits"].double().cpu().numpy()
    if case["scoring"] == "sigmoid":
        score = np.where(x >= 0, 1 / (1 + np.exp(-np.abs(x))), np.exp(-np.abs(x)) / (1 + np.exp(-np.abs(x))))
    else:
        score = np.exp(x - np.logaddexp.reduce(x, axis=1, keepdims=True))
    choice = score + (s["bias"].double().cpu().numpy() if case["bias"] else 0)
    if case["groups"] == 1 and not case["bias"]:
        choice = x                                          # scores rise with the logits
    groups = choice.reshape(len(x), case["groups"], -1)
    worth = np.partition(groups, -min(2, groups.shape[2]), axis=2)[..., -min(2, groups.shape[2]):].sum(2) if case["groups"] > 1 else groups.max(2)
    best = np.argsort(-worth, axis=1, kind="stable")[:, :case["top_groups"]]
    shut = np.ones(worth.shape, bool)
    np.put_along_axis(shut, best, False, axis=1)
    choice = np.where(np.repeat(shut, groups.shape[2], axis=1), -np.inf, choice)
    expert = np.argsort(-choice, axis=1, kind="stable")[:, :case["top"]]
    weights = np.take_along_axis(score, expert, axis=1)
    weights = case["scale"] * weights / weights.sum(1, keepdims=True)
    return {"token": np.repeat(np.arange(len(x), dtype=np.int32), case["top"]), "expert": expert.reshape(-1).astype(np.int32), "weights": weights}
