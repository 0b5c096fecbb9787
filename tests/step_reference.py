"""The operators of a decoder step in 64 bits, from their formulas, and how far a kernel may be from them."""
import numpy as np
import torch

U32 = 2.0 ** -24        # half a unit of a 32-bit sum or product


def half_unit(dtype) -> float:
    return torch.finfo(dtype).eps / 2


def paged_cache(lengths, page, kv_heads, dim, dtype, seed, layout="tokens", spare=3, rest=float("nan"), device="cuda:0"):
    """Caches whose used tokens are N(0, 1) and all else is `rest`, and a block table in random order: (k, v, table)."""
    g = torch.Generator().manual_seed(seed)
    have = [-(-n // page) for n in lengths]
    blocks, width = sum(have) + spare, max(have + [0]) + 2
    order = torch.randperm(blocks, generator=g)
    shape = (2, blocks, page, kv_heads, dim) if layout == "tokens" else (2, blocks, kv_heads, page, dim)
    cache = torch.full(shape, rest, dtype=dtype)
    if layout != "tokens":
        cache = cache.transpose(2, 3)
    table = torch.full((len(lengths), width), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(lengths):
        table[b, :have[b]] = order[at:at + have[b]].int()
        for j in range(have[b]):
            m = min(page, n - j * page)
            cache[:, order[at + j], :m] = torch.randn((2, m, kv_heads, dim), generator=g).to(dtype)
        at += have[b]
    moved = cache.to(device) if layout == "tokens" else cache.transpose(2, 3).contiguous().to(device).transpose(2, 3)
    return moved[0], moved[1], table.to(device)


def attention(q, k, v, table, lengths, scale):
    """(out, bound): the definition in 64 bits, and what the kernel's 32-bit sums and its rounding may be off by.

    Scores: dim products summed in 32 bits (a tensor core may drop instead of round: a whole unit each), one product with
    the scale and one exponential.  Their absolute error d makes every weight wrong by a factor of at most e^d, numerator and
    denominator alike; the weights are handed on as a sum of two 16-bit values (2^-16 of each, and 2^-24 of the largest one where the second is subnormal); values are summed
    in 32 bits, 16 tokens a step; parts are rescaled and joined a few times."""
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    bound = torch.zeros_like(out)
    share = q.shape[1] // k.shape[2]
    for b, n in enumerate(lengths):
        if n == 0:
            continue
        page = k.shape[1]
        blocks = table[b, :-(-n // page)].long()
        keys = k[blocks].flatten(0, 1)[:n].double().repeat_interleave(share, 1)
        values = v[blocks].flatten(0, 1)[:n].double().repeat_interleave(share, 1)
        x = q[b].double()
        s = torch.einsum("hd,thd->ht", x, keys) * scale
        p = torch.softmax(s, 1)
        out[b] = torch.einsum("ht,thd->hd", p, values)
        size = torch.einsum("hd,thd->ht", x.abs(), keys.abs()).amax(1) * abs(scale)
        d = (q.shape[2] + 4) * 2 * U32 * size + s.abs().amax(1) * 4 * U32 + 2.0 ** -21
        spread = torch.einsum("ht,thd->hd", p, values.abs())
        bound[b] = half_unit(q.dtype) * out[b].abs() + spread * (2 * d[:, None] + 2.0 ** -16 + (n / 16 + 64) * 4 * U32) \
            + n * p.amax(1)[:, None] * 2.0 ** -25 * values.abs().amax(0) + torch.finfo(q.dtype).tiny
    return out, bound


def qk_norm_rope(x, weight, eps, cos, sin, rotated, interleaved):
    """x [T][heads][dim] -> (values, magnitudes): in 64 bits; the magnitudes are sums of the terms' sizes."""
    y = x.double()
    if weight is not None:
        y = y / (y.square().mean(-1, keepdim=True) + eps).sqrt() * weight.double()
    size = y.abs()
    if rotated:
        half = rotated // 2
        c, s = cos.double()[:, None, :], sin.double()[:, None, :]
        pick = (slice(0, rotated, 2), slice(1, rotated, 2)) if interleaved else (slice(0, half), slice(half, rotated))
        a, b = y[..., pick[0]].clone(), y[..., pick[1]].clone()
        y, size = y.clone(), size.clone()
        y[..., pick[0]], y[..., pick[1]] = a * c - b * s, b * c + a * s
        size[..., pick[0]], size[..., pick[1]] = a.abs() * c.abs() + b.abs() * s.abs(), b.abs() * c.abs() + a.abs() * s.abs()
    return y, size


def qk_bound(y, size, dtype):
    """A mean of up to 256 squares in 32 bits, root, division, two products, then a rotation: each term is good to 32 units of 2^-24."""
    return half_unit(dtype) * y.abs() + size * 32 * U32 * (1 + half_unit(dtype)) + torch.finfo(dtype).tiny


def extend_tables(lengths, new, granted, table, page, blocks, tokens):
    """One request after another, as the header says it.  Returns everything, and whether something was left out."""
    lengths, new, granted, table = (np.asarray(x).astype(np.int64) for x in (lengths, new, granted, table))
    table = table.copy()
    positions, slots = np.zeros(tokens, np.int64), np.full(tokens, -1, np.int64)
    after, starts, row, share, used, bad = lengths.copy(), [0], 0, 0, 0, False
    for b, (n, m) in enumerate(zip(lengths, new)):
        added = max(int(m), 0)
        ok = n >= 0 and m >= 0 and n + m < 2 ** 31 and -(-(n + m) // page) <= table.shape[1] and (added == 0 or row + added <= tokens)
        fresh = int(-(-(n + m) // page) + (-n // page)) if ok else 0
        served = ok and (fresh == 0 or share + fresh <= len(granted))
        bad |= not served
        if served:
            first = -(-n // page)
            for j in range(fresh):
                e = granted[share + j]
                if not 0 <= e < blocks:
                    e, bad = -1, True
                table[b, first + j] = e
            for i in range(added):
                p = n + i
                e = table[b, p // page]
                positions[row + i] = p
                if 0 <= e < blocks:
                    slots[row + i] = e * page + p % page
                else:
                    bad = True
            after[b] = n + m
            if fresh:
                used = share + fresh
        row += added
        share += fresh
        starts.append(row)
    return {"lengths": after, "starts": np.minimum(starts, 2 ** 31 - 1), "positions": positions, "slots": slots, "used": np.array([used]), "table": table}, bad


def route(logits, top_k, bias, sigmoid, groups, top_groups, renormalise, scale):
    """(experts, weights) row by row; ties to the lower index."""
    x = np.asarray(logits, np.float64)
    T, E = x.shape
    size = E // groups
    experts, weights = np.empty((T, top_k), np.int64), np.empty((T, top_k))
    for t in range(T):
        with np.errstate(over="ignore"):
            s = 1 / (1 + np.exp(-x[t])) if sigmoid else np.exp(x[t] - x[t].max())
        if not sigmoid:
            s = s / s.sum()
        c = s if bias is None else s + np.asarray(bias, np.float64)
        kept = range(groups)
        if top_groups < groups:
            worth = [np.sort(c[g * size:(g + 1) * size])[-2:].sum() for g in range(groups)]
            kept = sorted(range(groups), key=lambda g: (-worth[g], g))[:top_groups]
        able = [e for g in sorted(kept) for e in range(g * size, (g + 1) * size)]
        best = sorted(able, key=lambda e: (-c[e], e))[:top_k]
        w = s[best]
        if renormalise:
            w = w / w.sum() if w.sum() > 0 else np.zeros_like(w)
        experts[t], weights[t] = best, w * scale
    return experts, weights
