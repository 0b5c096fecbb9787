"""GPU: norms of queries and keys, rotation and the cache write in one pass, against the formula in 64 bits."""
import pytest
import torch

import paper_2609_34380_b200 as dps
from paper_2609_34380_b200 import binding
from tests import step_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
FAR = 1000


def problem(T, heads, kv_heads, dim, page, dtype, rotated, norm, seed, padding=(), layout="tokens"):
    g = torch.Generator().manual_seed(seed)
    qkv = (torch.randn((T, (heads + 2 * kv_heads) * dim), generator=g) * 3).to(dtype).to(DEV)
    blocks = -(-T // page) + 2
    shape = (2, blocks, page, kv_heads, dim) if layout == "tokens" else (2, blocks, kv_heads, page, dim)
    cache = torch.full(shape, 5.0, dtype=dtype, device=DEV)
    if layout != "tokens":
        cache = cache.transpose(2, 3)
    slots = torch.randperm(blocks * page, generator=g)[:T]
    slots[list(padding)] = -1
    positions = torch.randint(0, FAR, (T,), generator=g, dtype=torch.int32)
    half = rotated // 2
    angle = torch.arange(FAR, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(half, dtype=torch.float64) / max(half, 1))
    cos_sin = torch.cat([angle.cos(), angle.sin()], 1).float().to(DEV) if rotated else None
    w = [torch.randn((dim,), generator=g).to(dtype).to(DEV) for _ in range(2)] if norm else [None, None]
    return qkv, cache[0], cache[1], slots.to(DEV), positions.to(DEV), cos_sin, w[0], w[1]


def check(p, q, heads, kv_heads, dim, eps, interleaved, filled=5.0):
    qkv, k_cache, v_cache, slots, positions, cos_sin, qw, kw = p
    x = qkv.view(-1, heads + 2 * kv_heads, dim) if qkv.is_contiguous() else qkv.reshape(-1, heads + 2 * kv_heads, dim)
    live = slots >= 0
    rotated = 0 if cos_sin is None else cos_sin.shape[1]
    row = cos_sin[positions.long()] if rotated else torch.zeros((x.shape[0], 0), device=DEV)
    cos, sin = row[:, :rotated // 2], row[:, rotated // 2:]
    page = k_cache.shape[1]
    at = slots[live]
    for got, part, w in ((q[live], x[:, :heads], qw), (k_cache[at // page, at % page], x[:, heads:heads + kv_heads], kw)):
        y, size = ref.qk_norm_rope(part, w, eps, cos, sin, rotated, interleaved)
        off = (got.double() - y[live]).abs()
        assert bool((off <= ref.qk_bound(y, size, qkv.dtype)[live]).all()), float((off / ref.qk_bound(y, size, qkv.dtype)[live]).max())
    assert torch.equal(v_cache[at // page, at % page], x[live][:, heads + kv_heads:])
    rest = torch.ones(k_cache.shape[0] * page, dtype=torch.bool, device=DEV)
    rest[at] = False
    for c in (k_cache, v_cache):                             # all other tokens as they were
        other = c.reshape(-1, kv_heads, dim)[rest]
        assert bool((other == filled).all())


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("T,heads,kv_heads,dim,page,rotated,norm", [
    (1, 4, 4, 128, 16, 128, True), (5, 8, 2, 128, 16, 64, False), (33, 6, 2, 64, 8, 64, True), (7, 9, 3, 96, 24, 32, True), (3, 5, 5, 80, 7, 80, False),
    (9, 3, 1, 256, 16, 256, True), (4, 4, 2, 192, 1, 160, True), (130, 1, 1, 64, 64, 16, True), (2, 2, 2, 8, 4, 0, True), (6, 7, 1, 40, 3, 32, True),
    (3, 32, 8, 128, 16, 0, False), (2, 0, 3, 64, 16, 64, True), (257, 17, 1, 16, 5, 16, True)])
def test_against_the_formula(dtype, interleaved, T, heads, kv_heads, dim, page, rotated, norm):
    p = problem(T, heads, kv_heads, dim, page, dtype, rotated, norm, 7, padding=[T // 2] if T > 4 else [])
    q = torch.full((T, heads, dim), 3.0, dtype=dtype, device=DEV)
    assert dps.dps_qk_norm_rope(*p, eps=1e-5, interleaved=interleaved, q_out=q) is q
    check(p, q, heads, kv_heads, dim, 1e-5, interleaved)
    if T > 4:
        assert bool((q[T // 2] == 3.0).all())                # padding: left alone
    assert dps.dps_stream_status() == dps.DPS_OK


@pytest.mark.parametrize("layout", ["tokens", "heads"])
def test_strides_and_queries_in_place(layout):
    heads, kv_heads, dim = 8, 2, 64
    p = list(problem(19, heads, kv_heads, dim, 8, torch.float16, 64, True, 8, layout=layout))
    dense = p[0].clone()
    wide = torch.full((19, 12 * 64 + 40), float("nan"), dtype=torch.float16, device=DEV)
    p[0] = wide[:, 16:16 + 12 * 64]
    p[0].copy_(dense)
    q = p[0][:, :heads * dim].unflatten(1, (heads, dim))     # over the queries themselves
    assert q.data_ptr() == p[0].data_ptr()
    dps.dps_qk_norm_rope(*p, q_out=q)
    check([dense, *p[1:]], q, heads, kv_heads, dim, 1e-6, False)
    assert torch.equal(p[0][:, heads * dim:], dense[:, heads * dim:]) and bool(torch.isnan(wide[:, :16]).all()) and bool(torch.isnan(wide[:, -24:]).all())
    assert dps.dps_stream_status() == dps.DPS_OK


def test_plain_rows_instead_of_pages():
    T, heads, kv_heads, dim = 21, 4, 2, 128
    p = problem(T, heads, kv_heads, dim, 16, torch.bfloat16, 128, True, 9)
    k, v = (torch.full((T, 1, kv_heads, dim), 5.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    p = (p[0], k, v, torch.arange(T, device=DEV), *p[4:])
    check(p, dps.dps_qk_norm_rope(*p), heads, kv_heads, dim, 1e-6, False)


def test_rows_that_are_left_out():
    heads, kv_heads, dim, page = 4, 2, 64, 8
    for field, value in [(3, 10 ** 6), (3, 2 ** 40), (4, -1), (4, FAR)]:
        p = list(problem(6, heads, kv_heads, dim, page, torch.float16, 64, True, 10))
        bad = p[field].clone()
        bad[2] = value
        broken = [*p]
        broken[field] = bad
        q = torch.full((6, heads, dim), 3.0, dtype=torch.float16, device=DEV)
        dps.dps_qk_norm_rope(*broken, q_out=q)
        assert dps.dps_stream_status() == binding.DPS_ERR_DATA and dps.dps_stream_status() == dps.DPS_OK
        assert bool((q[2] == 3.0).all())
        p[3] = p[3].clone()
        p[3][2] = -1
        check(p, q, heads, kv_heads, dim, 1e-6, False)


def test_rows_of_zeros_and_of_large_values():
    p = list(problem(4, 2, 2, 64, 8, torch.float16, 64, True, 12))
    p[0][0] = 0
    p[0][1] = 60000.0                                        # squares beyond FP16, not beyond 32 bits
    p[0][2] = 2.0 ** -24
    q = dps.dps_qk_norm_rope(*p, eps=1e-6)
    check(p, q, 2, 2, 64, 1e-6, False)
    assert not bool(q[0].any())


def test_far_slots():
    """Slots whose elements start beyond 2^31, in a cache of 4.6 GB."""
    p = problem(5, 2, 8, 128, 16, torch.float16, 128, True, 13)
    want = dps.dps_qk_norm_rope(*p)
    k = torch.empty((140000, 16, 8, 128), dtype=torch.float16, device=DEV)
    v = torch.empty_like(k)
    far = p[3] + (140000 - p[1].shape[0]) * 16
    got = dps.dps_qk_norm_rope(p[0], k, v, far, *p[4:])
    n = p[1].shape[0]
    assert torch.equal(got, want)
    for t in range(5):
        s, f = int(p[3][t]), int(far[t])
        assert f * 1024 > 2 ** 31
        assert torch.equal(k[f // 16, f % 16], p[1][s // 16, s % 16]) and torch.equal(v[f // 16, f % 16], p[2][s // 16, s % 16])
    assert n < 16


def test_captured_replayed_and_on_another_stream():
    heads, kv_heads, dim = 4, 2, 128
    p = problem(10, heads, kv_heads, dim, 16, torch.float16, 128, True, 14)
    q = torch.zeros((10, heads, dim), dtype=torch.float16, device=DEV)
    dps.dps_qk_norm_rope(*p, q_out=q)
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        dps.dps_qk_norm_rope(*p, q_out=q)
    p[0].normal_()
    p[3].copy_(torch.randperm(10))
    p[4].copy_(torch.randint(0, FAR, (10,), dtype=torch.int32))
    p[1].fill_(5.0), p[2].fill_(5.0)
    graph.replay()
    check(p, q, heads, kv_heads, dim, 1e-6, False)
    with torch.cuda.stream(side):
        torch.cuda._sleep(10_000_000)
        q.zero_()
        p[1].fill_(5.0), p[2].fill_(5.0)
        dps.dps_qk_norm_rope(*p, q_out=q)
    again = dps.dps_qk_norm_rope(*p, stream=side)
    side.synchronize()
    check(p, q, heads, kv_heads, dim, 1e-6, False)
    assert torch.equal(again, q)


def test_refusals():
    p = problem(4, 4, 2, 64, 8, torch.float16, 64, True, 15)
    qkv, k, v, slots, positions, cos_sin, qw, kw = p
    launches = dps.dps_launch_count()
    for args, more, error in [
            ((qkv[:, :-64], k, v, slots, positions, cos_sin, qw, kw[:32]), {}, ValueError), ((qkv[:, :-8], k, v, slots), {}, ValueError),
            ((qkv[:, :128], k, v, slots), {}, ValueError), ((qkv.bfloat16(), k, v, slots), {}, TypeError), ((qkv.float(), k, v, slots), {}, TypeError),
            ((qkv, k, v, slots.int()), {}, TypeError), ((qkv, k, v, slots[:3]), {}, ValueError), ((qkv, k, v, slots, positions.long(), cos_sin), {}, TypeError),
            ((qkv, k, v, slots, positions, cos_sin.half()), {}, TypeError), ((qkv, k, v, slots, None, cos_sin), {}, dps.DpsError),
            ((qkv, k, v, slots, positions, cos_sin[:, :24].contiguous()), {}, dps.DpsError), ((qkv, k, v, slots, positions, cos_sin, qw, None), {}, dps.DpsError),
            ((qkv, k, v, slots, positions, cos_sin, qw.float(), kw), {}, TypeError), ((qkv, k, v, slots), {"eps": -1.0}, dps.DpsError),
            ((qkv, k, v, slots), {"q_out": torch.empty((4, 5, 64), dtype=torch.float16, device=DEV)}, ValueError),
            ((qkv, k, v, slots), {"q_out": torch.empty((4, 64, 4), dtype=torch.float16, device=DEV).transpose(1, 2)}, ValueError),
            ((qkv, k, v, slots.cpu()), {}, ValueError), ((qkv, k[..., :60], v[..., :60], slots), {}, ValueError)]:
        with pytest.raises(error):
            dps.dps_qk_norm_rope(*args, **more)
    assert dps.dps_launch_count() == launches
    assert dps.dps_qk_norm_rope(qkv[:0], k, v, slots[:0]).shape == (0, 4, 64)
    assert binding._native.qk_norm_rope(qkv, k, v, slots, positions, cos_sin, qw, kw, 1e-6, False, None) is not None
