"""GPU: the operators between the linears as a server runs them -- blocks from the shared-region manager, block tables, norms and rotation with
the cache write, attention, routing into the grouped linear."""
import numpy as np
import pytest
import torch

import paper_2609_34380_b200 as dps
from paper_2609_34380_b200 import sum_manager as sm, workloads
from paper_2609_34380_b200.kv_cache import PagedKvCache
from tests import step_reference as ref
from tests.helpers import split_both

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HEADS, KV_HEADS, DIM, PAGE = 8, 2, 64, 16


def rotation(positions):
    angle = torch.arange(positions, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(DIM // 2, dtype=torch.float64) / (DIM // 2))
    return torch.cat([angle.cos(), angle.sin()], 1).float().to(DEV)


def test_requests_come_and_go():
    """Prompts, decode steps, finished requests, a manager that gives up residual units: attention against each request's own history."""
    mgr = sm.SumManager(units=7, blocks_per_unit=3, residual_tensors=5)
    cache = PagedKvCache(mgr, 2, HEADS, KV_HEADS, DIM, PAGE, max_requests=7, max_tokens_per_request=200)
    rng, cos_sin = np.random.default_rng(3), rotation(256)
    history = []                                            # per row: the keys and values of its tokens, as the cache holds them
    refused = fast = checked = 0
    for step_number in range(90):
        while len(history) < 7 and rng.random() < 0.5:
            assert cache.admit() == len(history)
            history.append([[], []])
        if not history:
            continue
        single = step_number % 3 != 0 and all(len(h[0]) for h in history)
        new = [1 if single else int(rng.integers(0, 40)) if not h[0] else int(rng.integers(0, 3)) for h in history]
        if any(n + m > 200 for n, m in zip(cache.lengths, new)):
            with pytest.raises(ValueError):
                cache.extend([m + 208 for m in new])
            step = None
        else:
            step = cache.extend(new, rows=sum(new) + 5)
            refused += step is None
        mgr.check()
        fast += mgr.mode == sm.MODE_FAST
        if step is None:                                    # no room: the longest request goes
            row = int(np.argmax(cache.lengths))
            moved = cache.finish(row)
            if moved is None:
                history.pop()
            else:
                history[row] = history.pop()
            continue
        assert step.lengths.tolist() == cache.lengths and step.tokens == sum(new)
        for layer in range(2):
            qkv = torch.randn((sum(new) + 5, (HEADS + 2 * KV_HEADS) * DIM), device=DEV).half()
            q = cache.write(layer, step, qkv, cos_sin)
            if layer == 0:                                  # where did they go: read the rows back through the slots
                k, v = (c.view(-1, KV_HEADS, DIM) for c in cache.caches[0])
                at = 0
                for b, m in enumerate(new):
                    for t in range(at, at + m):
                        slot = int(step.slots[t])
                        assert int(step.positions[t]) == len(history[b][0])
                        history[b][0].append(k[slot].clone())
                        history[b][1].append(v[slot].clone())
                        assert torch.equal(v[slot].flatten(), qkv[t, (HEADS + KV_HEADS) * DIM:])
                    at += m
                if step.single:
                    out = cache.attend(0, step, q)
                    for b, (keys, values) in enumerate(history):
                        n = len(keys)
                        page = torch.stack(keys)[None], torch.stack(values)[None]
                        want, bound = ref.attention(q[b:b + 1], *page, torch.zeros((1, 1), dtype=torch.int32, device=DEV), [n], DIM ** -0.5)
                        assert bool(((out[b:b + 1].double() - want).abs() <= bound).all()), (step_number, b)
                        checked += 1
        assert dps.dps_stream_status() == dps.DPS_OK
        if rng.random() < 0.15 and len(history) > 1:
            row = int(rng.integers(len(history)))
            moved = cache.finish(row)
            if moved is None:
                history.pop()
            else:
                history[row] = history.pop()
    assert checked > 50 and fast > 5 and refused > 0, (checked, fast, refused)
    while history:
        cache.finish(0)
        history.pop()
    mgr.check()
    assert mgr.kv_blocks_in_use == 0 and cache.lengths == []


def test_refusals():
    cache = PagedKvCache(sm.SumManager(2, 4, 0), 1, 4, 4, DIM, PAGE, max_requests=2, max_tokens_per_request=40)
    cache.admit(), cache.admit()
    with pytest.raises(ValueError):
        cache.admit()
    for new, kw in (([1], {}), ([1, -1], {}), ([1, 49], {}), ([5, 5], {"rows": 9})):
        with pytest.raises(ValueError):
            cache.extend(new, **kw)
    for row in (-1, 2):
        with pytest.raises(ValueError):
            cache.finish(row)
    assert cache.lengths == [0, 0]
    assert cache.extend([40, 40]) is not None and cache.extend([8, 8]) is not None
    cache.finish(0)
    step = cache.extend([0])
    assert step.tokens == 0 and not step.single
    with pytest.raises(ValueError):
        cache.attend(0, step, torch.zeros((1, 4, DIM), dtype=torch.float16, device=DEV))


def test_no_requests_and_no_tokens():
    cache = PagedKvCache(sm.SumManager(2, 4, 0), 1, 4, 4, DIM, PAGE, max_requests=2, max_tokens_per_request=40)
    for rows in (0, 3):
        step = cache.extend([], rows=rows)
        assert step.tokens == 0 and step.slots.tolist() == [-1] * rows and step.starts.tolist() == [0]
        q = cache.write(0, step, torch.ones((rows, 12 * DIM), dtype=torch.float16, device=DEV))
        assert q.shape == (rows, 4, DIM) and cache.attend(0, step, q).shape == (0, 4, DIM)
    cache.admit()
    step = cache.extend([0], rows=2)
    cache.write(0, step, torch.ones((2, 12 * DIM), dtype=torch.float16, device=DEV))
    assert step.lengths.tolist() == [0] and not bool(cache.caches.any()) and dps.dps_stream_status() == dps.DPS_OK


def test_a_decoder_step_in_one_graph():
    """QKV linear, norm and rotation, attention, O linear, router, gate/up of the experts: captured once, replayed on other data; each replay equals the
    calls made one by one, and the routed rows are the experts' own linears."""
    hidden, experts, ffn, n = 512, 8, 256, 5
    planes = {name: split_both(workloads.weights(rows, hidden, 700 + i), dps.DPS_ENC_AUTO)[:3]
              for i, (name, rows) in enumerate({"qkv": (HEADS + 2 * KV_HEADS) * DIM, "o": hidden, "router": experts}.items())}
    moe = [split_both(workloads.weights(ffn, hidden, 720 + e), dps.DPS_ENC_E5M2)[:2] for e in range(experts)]
    mp, mr = torch.stack([m[0] for m in moe]), torch.stack([m[1] for m in moe])
    encs = [dps.DPS_ENC_E5M2] * experts
    cache = PagedKvCache(sm.SumManager(8, 8, 0), 1, HEADS, KV_HEADS, DIM, PAGE, max_requests=n, max_tokens_per_request=64)
    cos_sin, weight = rotation(128), torch.rand(DIM, device=DEV).half() + 0.5
    bias = torch.randn(experts, device=DEV) * 0.1
    for _ in range(n):
        cache.admit()
    prompt = cache.extend([3, 20, 1, 16, 31])
    cache.write(0, prompt, torch.randn((71, (HEADS + 2 * KV_HEADS) * DIM), device=DEV).half(), cos_sin, weight, weight)
    k, v = cache.caches[0]
    ws = torch.empty(dps.dps_moe_workspace_bytes(2 * n, experts, hidden), dtype=torch.uint8, device=DEV)

    def linear(name, x):
        p, r, enc = planes[name]
        return dps.dps_linear(dps.DPS_MODE_FULL, enc, x, p, r)

    def layer(x, lengths, new, granted, table, after, starts, positions, slots, used):
        dps.dps_extend_block_tables(lengths, new, granted, table, PAGE, cache.blocks, after, starts, positions, slots, used)
        q = dps.dps_qk_norm_rope(linear("qkv", x), k, v, slots, positions, cos_sin, weight, weight)
        h = linear("o", dps.dps_paged_attention(q, k, v, table, after, workspace=cache.workspace).view(n, hidden))
        token, expert, share = dps.dps_route_experts(linear("router", h), 2, bias, dps.DPS_SCORE_SIGMOID)
        return q, h, token, expert, share, dps.dps_moe_linear(dps.DPS_MODE_FULL, encs, h, token, expert, mp, mr, workspace=ws)

    new = torch.ones(n, dtype=torch.int32, device=DEV)
    i32 = lambda size: torch.zeros(size, dtype=torch.int32, device=DEV)  # noqa: E731
    state = dict(lengths=cache._lengths[cache._now, :n].clone(), new=new, granted=i32(8), table=cache.block_table.clone(), after=i32(n), starts=i32(n + 1),
                 positions=i32(n), slots=torch.zeros(n, dtype=torch.int64, device=DEV), used=i32(1))
    free = [b for b in range(cache.blocks) if b not in set(cache.block_table.flatten().tolist())]
    x = torch.randn((n, hidden), device=DEV).half()
    state["granted"].copy_(torch.tensor(free[:8], dtype=torch.int32))
    snapshot = [cache.caches.clone(), state["table"].clone()]
    layer(x, **state)                                       # (first calls set up what a capture may not)
    torch.cuda.synchronize()
    cache.caches.copy_(snapshot[0]), state["table"].copy_(snapshot[1])
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        out = layer(x, **state)
    cache.caches.copy_(snapshot[0]), state["table"].copy_(snapshot[1])
    granted = 0
    for step in range(20):
        x.copy_(torch.randn((n, hidden), device=DEV).half())
        state["granted"].copy_(torch.tensor((free[granted:] + [0] * 8)[:8], dtype=torch.int32))
        before = [cache.caches.clone(), state["table"].clone()]
        want = [t.clone() for t in layer(x, **state)]
        written = [cache.caches.clone(), state["table"].clone()]
        cache.caches.copy_(before[0]), state["table"].copy_(before[1])
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b), step
        assert torch.equal(cache.caches, written[0]) and torch.equal(state["table"], written[1])
        # the attention in it against the definition, and the experts' rows against their own linears
        q, h, token, expert, share, rows = out
        attended = dps.dps_paged_attention(q, k, v, state["table"], state["after"], workspace=cache.workspace)
        exact, bound = ref.attention(q, k, v, state["table"], state["after"].tolist(), DIM ** -0.5)
        assert bool(((attended.double() - exact).abs() <= bound).all())
        experts_want, weights_want = ref.route(linear("router", h).double().cpu().numpy(), 2, bias.double().cpu().numpy(), True, 1, 1, True, 1.0)
        assert np.array_equal(expert.view(n, 2).cpu().numpy(), experts_want)
        assert np.allclose(share.cpu().numpy(), weights_want, rtol=64 * ref.U32)
        for a in range(2 * n):
            e = int(expert[a])
            one = dps.dps_linear(dps.DPS_MODE_FULL, encs[e], h[int(token[a])][None].contiguous(), mp[e].contiguous(), mr[e].contiguous())
            assert torch.allclose(rows[a].float(), one[0].float(), rtol=2e-3, atol=2e-3 * float(one.abs().max()))
        granted += int(state["used"])
        state["lengths"].copy_(state["after"])
    assert granted > 3 and dps.dps_stream_status() == dps.DPS_OK
