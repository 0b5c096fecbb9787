"""GPU: attention of one new token over a paged cache, against the definition in 64 bits."""
import ctypes

import pytest
import torch

import paper_2609_34380_b200 as dps
from paper_2609_34380_b200 import binding
from tests import step_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def problem(lengths, heads, kv_heads, dim, page, dtype, seed, layout="tokens"):
    k, v, table = ref.paged_cache(lengths, page, kv_heads, dim, dtype, seed, layout)
    g = torch.Generator().manual_seed(seed + 1)
    q = torch.randn((len(lengths), heads, dim), generator=g).to(dtype).to(DEV)
    return q, k, v, table, torch.tensor(lengths, dtype=torch.int32, device=DEV)


def check(got, q, k, v, table, lengths, scale=None, what=""):
    want, bound = ref.attention(q, k, v, table, lengths.tolist(), q.shape[2] ** -0.5 if scale is None else scale)
    off = (got.double() - want).abs()
    assert bool(torch.isfinite(got).all()), what
    assert bool((off <= bound).all()), (what, float((off / bound).max()))


EDGES = [0, 1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 127, 128, 129, 0, 255, 257, 300]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("heads,kv_heads,dim,page", [(4, 4, 128, 16), (8, 1, 128, 16), (6, 2, 64, 8), (9, 3, 96, 24), (5, 5, 80, 7), (16, 1, 128, 32),
                                                     (12, 1, 64, 5), (20, 1, 128, 16), (34, 2, 40, 128), (4, 2, 256, 16), (12, 1, 256, 64), (3, 1, 192, 1),
                                                     (2, 2, 8, 16)])
def test_lengths_around_every_edge(dtype, heads, kv_heads, dim, page):
    p = problem(EDGES, heads, kv_heads, dim, page, dtype, 11)
    got = dps.dps_paged_attention(*p)
    check(got, *p)
    assert not bool(got[0].any()) and not bool(got[14].any())               # no tokens: zeros
    assert dps.dps_stream_status() == dps.DPS_OK


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("lengths,heads,kv_heads,dim,page", [
    ([20011], 8, 1, 128, 16), ([1, 9000, 0, 40, 700], 8, 2, 128, 48), ([5000] * 3, 16, 1, 64, 16), ([2500, 1], 3, 3, 256, 32), ([19000], 1, 1, 96, 64),
    ([100, 4000, 3], 24, 1, 128, 16)])
def test_split_over_the_length(dtype, lengths, heads, kv_heads, dim, page):
    p = problem(lengths, heads, kv_heads, dim, page, dtype, 21)
    ws = dps.dps_paged_attention_workspace(heads, kv_heads, dim)
    got = dps.dps_paged_attention(*p, workspace=ws)
    check(got, *p)
    again = dps.dps_paged_attention(*p, workspace=ws)                        # the workspace is ready again, and the parts are joined in their order
    assert torch.equal(got.view(torch.int16), again.view(torch.int16))
    assert dps.dps_stream_status() == dps.DPS_OK


def test_many_requests():
    lengths = [(37 * i * i) % 211 for i in range(700)]
    p = problem(lengths, 4, 2, 64, 16, torch.float16, 31)
    check(dps.dps_paged_attention(*p), *p)
    none = problem([0] * 5, 4, 2, 64, 16, torch.float16, 32)
    assert not bool(dps.dps_paged_attention(*none).any())
    q, k, v, table, n = none
    assert dps.dps_paged_attention(q[:0], k, v, table[:0], n[:0]).shape == (0, 4, 64)
    assert not bool(dps.dps_paged_attention(q, k, v, table[:, :0], n).any())
    assert dps.dps_stream_status() == dps.DPS_OK


@pytest.mark.parametrize("layout", ["tokens", "heads"])
def test_strides(layout):
    """Queries inside the QKV linear's output, either order of the cache, a cache inside a larger one, a table inside a larger one."""
    lengths = [70, 1, 333]
    q, k, v, table, n = problem(lengths, 8, 2, 128, 16, torch.float16, 41, layout)
    qkv = torch.full((3, 12 * 128), float("nan"), dtype=torch.float16, device=DEV)
    inside = qkv[:, :1024].view(3, 8, 128)
    inside.copy_(q)
    wide = torch.full((3, table.shape[1] + 5), 1 << 30, dtype=torch.int32, device=DEV)
    wide[:, 2:-3] = table
    got = dps.dps_paged_attention(inside, k, v, wide[:, 2:-3], n)
    check(got, q, k, v, table, n)
    turned = q.transpose(1, 2).contiguous().transpose(1, 2)                  # a last dimension that is not dense is refused
    with pytest.raises(ValueError):
        dps.dps_paged_attention(turned, k, v, table, n)
    both = torch.full((2, k.shape[0], 2, 16, 3, 128), float("nan"), dtype=torch.float16, device=DEV)     # layers side by side, a head too many
    both[:, :, 1, :, :2] = torch.stack([k, v])
    kk, vv = both[0, :, 1, :, :2], both[1, :, 1, :, :2]
    assert torch.equal(dps.dps_paged_attention(q, kk, vv, table, n), got)
    # heads of a request behind one another in another order of memory
    other = torch.empty((8, 3, 128), dtype=torch.float16, device=DEV).transpose(0, 1)
    other.copy_(q)
    assert torch.equal(dps.dps_paged_attention(other, k, v, table, n), got)
    assert dps.dps_stream_status() == dps.DPS_OK


def test_scales_and_extreme_scores():
    q, k, v, table, n = problem([200, 77], 8, 8, 64, 16, torch.float16, 51)
    for scale in (0.0, -0.3, 2.0):
        check(dps.dps_paged_attention(q, k, v, table, n, scale=scale), q, k, v, table, n, scale)
    big = (q * 60).clamp(-2000, 2000)                                        # weights that are all but one-hot
    check(dps.dps_paged_attention(big, k, v, table, n), big, k, v, table, n)
    # one key far above the rest at the very end, another at the very start: the running maximum moves late, or never
    for at in (199, 0):
        k2 = k.clone()
        k2[table[0, at // 16].long(), at % 16] = 8 * q[0]
        check(dps.dps_paged_attention(q, k2, v, table, n), q, k2, v, table, n)


def test_infinite_values_follow_the_formula():
    q, k, v, table, n = problem([40], 1, 1, 64, 16, torch.float16, 52)
    k2 = k.clone()
    k2[table[0, 1].long(), 3] = float("inf")                                 # a score of +Inf or NaN: the softmax has no value
    assert bool(torch.isnan(dps.dps_paged_attention(q.abs(), k2, v, table, n)).all())
    k2[table[0, 1].long(), 3] = float("-inf")                                # a score of -Inf: the token has no weight
    got = dps.dps_paged_attention(q.abs() + 0.1, k2, v, table, n)
    k3, keep = k2.clone(), [t for t in range(40) if t != 19]
    flat = lambda c: c[table[0, :3].long()].flatten(0, 1)[keep, 0].double()  # noqa: E731
    w = torch.softmax(flat(k3) @ (q.abs() + 0.1)[0, 0].double() / 8, 0)
    assert float((got[0, 0].double() - w @ flat(v)).abs().max()) < 2e-3


def test_far_offsets():
    """Blocks that start beyond 2^32 bytes and 2^31 elements of the cache."""
    blocks, page, kv_heads, dim = 140000, 16, 8, 128                        # 4.6 GB each
    k = torch.empty((blocks, page, kv_heads, dim), dtype=torch.float16, device=DEV)
    v = torch.empty_like(k)
    lengths = [100, 37]
    small = problem(lengths, 8, kv_heads, dim, page, torch.float16, 61)
    q, ks, vs, table, n = small
    far = torch.where(table >= 0, blocks - 1 - table, table)
    for i in range(ks.shape[0]):
        k[blocks - 1 - i], v[blocks - 1 - i] = ks[i], vs[i]
    assert (blocks - 20) * page * kv_heads * dim > 2 ** 31
    assert torch.equal(dps.dps_paged_attention(q, k, v, far, n), dps.dps_paged_attention(*small))


def test_bad_pages_and_lengths():
    q, k, v, table, n = problem([50, 20, 70], 4, 2, 64, 16, torch.float16, 71)
    want = dps.dps_paged_attention(q, k, v, table, n)
    assert dps.dps_stream_status() == dps.DPS_OK
    for bad in (-1, k.shape[0], 2 ** 31 - 1, -2 ** 31):
        broken = table.clone()
        broken[0, 1] = bad
        got = dps.dps_paged_attention(q, k, v, broken, n)
        assert dps.dps_stream_status() == binding.DPS_ERR_DATA
        assert dps.dps_stream_status() == dps.DPS_OK                         # reading clears it
        assert torch.equal(got[1:], want[1:])
        # the first request's other tokens still count
        page0, page2, page3 = (table[0, i].long() for i in (0, 2, 3))
        keys, values = (torch.cat([c[page0], c[page2], c[page3][:2]]).double() for c in (k, v))
        w = torch.softmax(torch.einsum("hd,thd->ht", q[0].double() / 8, keys.repeat_interleave(2, 1)), 1)
        assert float((got[0].double() - torch.einsum("ht,thd->hd", w, values.repeat_interleave(2, 1))).abs().max()) < 2e-3
    wrong = n.clone()
    wrong[1] = -5
    got = dps.dps_paged_attention(q, k, v, table, wrong)
    assert dps.dps_stream_status() == binding.DPS_ERR_DATA
    assert not bool(got[1].any()) and torch.equal(got[0], want[0]) and torch.equal(got[2], want[2])
    short = table[:, :2].contiguous()                                        # 32 tokens at most
    got = dps.dps_paged_attention(q, k, v, short, n)
    assert dps.dps_stream_status() == binding.DPS_ERR_DATA
    assert torch.equal(got, dps.dps_paged_attention(q, k, v, short, n.clamp(max=32)))
    assert dps.dps_stream_status() == dps.DPS_OK


def test_a_workspace_that_was_not_prepared():
    p = problem([50, 20], 4, 2, 64, 16, torch.float16, 81)
    need = dps.dps_paged_attention_workspace_bytes(4, 2, 64)
    ws = torch.randint(0, 256, (need,), dtype=torch.uint8, device=DEV)
    out = torch.full_like(p[0], 7.0)
    dps.dps_paged_attention(*p, out=out, workspace=ws)
    assert dps.dps_stream_status() == binding.DPS_ERR_WORKSPACE and bool((out == 7.0).all())
    dps.dps_paged_attention_workspace_init(ws)
    assert dps.dps_paged_attention(*p, out=out, workspace=ws) is out
    check(out, *p)
    with pytest.raises(dps.DpsError) as caught:
        dps.dps_paged_attention(*p, workspace=ws[:need - 16])
    assert caught.value.status == binding.DPS_ERR_WORKSPACE


def test_one_workspace_for_layers_of_several_shapes():
    shapes = [([4000], 8, 1, 128, 16), ([10, 20], 4, 4, 64, 16), ([3000, 2], 4, 1, 256, 16), ([2000], 16, 1, 128, 32), ([1] * 40, 2, 2, 64, 8)]
    need = max(dps.dps_paged_attention_workspace_bytes(h, kv, d) for _, h, kv, d, _ in shapes)
    ws = dps.dps_paged_attention_workspace_init(torch.empty(need, dtype=torch.uint8, device=DEV))
    for turn in range(2):
        for i, s in enumerate(shapes):
            p = problem(*s, torch.bfloat16, 90 + i)
            check(dps.dps_paged_attention(*p, workspace=ws), *p, what=f"{turn} {s}")


def test_captured_and_replayed_with_other_lengths():
    """The lengths are on the device: one graph serves every step."""
    lengths = [900, 0, 64, 2000]
    q, k, v, table, n = problem(lengths, 8, 2, 128, 16, torch.float16, 101)
    ws, out = dps.dps_paged_attention_workspace(8, 2, 128), torch.empty_like(q)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    dps.dps_paged_attention(q, k, v, table, n, out=out, workspace=ws)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        dps.dps_paged_attention(q, k, v, table, n, out=out, workspace=ws)
    for now in (lengths, [1, 0, 3, 1999], [0, 0, 0, 0], [900, 0, 64, 17]):
        n.copy_(torch.tensor(now, dtype=torch.int32))
        out.fill_(3.0)
        graph.replay()
        check(out, q, k, v, table, n, what=str(now))
    assert dps.dps_stream_status() == dps.DPS_OK


def test_streams():
    p = problem([700, 31], 8, 8, 64, 16, torch.float16, 111)
    want = dps.dps_paged_attention(*p)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    late = torch.zeros_like(p[0])
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
        late.copy_(p[0])
        got = dps.dps_paged_attention(late, *p[1:], workspace=dps.dps_paged_attention_workspace(8, 8, 64))
    other = dps.dps_paged_attention(*p, stream=side)                         # the ctypes way, on a named stream, making its own workspace
    by_handle = dps.dps_paged_attention(*p, stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(got, want) and torch.equal(other, want) and torch.equal(by_handle, want)


def test_nothing_beside_the_output_is_written():
    q, k, v, table, n = problem([100, 5000], 4, 1, 80, 16, torch.float16, 121)
    out = torch.full((4, 4, 80), 9.0, dtype=torch.float16, device=DEV)
    need = dps.dps_paged_attention_workspace_bytes(4, 1, 80)
    ws = torch.full((need + 256,), 0xA5, dtype=torch.uint8, device=DEV)
    dps.dps_paged_attention_workspace_init(ws[:need])
    before = [t.clone() for t in (q, k, v, table, n)]
    dps.dps_paged_attention(q, k, v, table, n, out=out[1:3], workspace=ws[:need])
    check(out[1:3], q, k, v, table, n)
    assert bool((out[0] == 9.0).all()) and bool((out[3] == 9.0).all()) and bool((ws[need:] == 0xA5).all())
    for a, b in zip((q, k, v, table, n), before):
        assert torch.equal(a.view(torch.uint8) if a.dtype is not torch.int32 else a, b.view(torch.uint8) if b.dtype is not torch.int32 else b)


def test_refusals():
    q, k, v, table, n = problem([50, 20], 4, 2, 64, 16, torch.float16, 131)
    ws = dps.dps_paged_attention_workspace(4, 2, 64)
    launches = dps.dps_launch_count()
    for args, kw, error in [
            ((q.float(), k, v, table, n), {}, TypeError), ((q.bfloat16(), k, v, table, n), {}, TypeError), ((q.cpu(), k, v, table, n), {}, ValueError),
            ((q, k, v[:-1], table, n), {}, ValueError), ((q, k.bfloat16(), v, table, n), {}, ValueError), ((q, k, v, table.long(), n), {}, TypeError),
            ((q, k, v, table[:1], n), {}, ValueError), ((q, k, v, table, n.long()), {}, TypeError), ((q, k, v, table, n[:1]), {}, ValueError),
            ((q[..., :32], k, v, table, n), {}, ValueError), ((q[:, :3], k, v, table, n), {}, dps.DpsError), ((q, k, v, table, n), {"out": q[:1]}, ValueError),
            ((q, k, v, table, n), {"out": torch.empty_like(q, dtype=torch.float32)}, TypeError), ((q, k, v, table, n), {"scale": float("nan")}, dps.DpsError),
            ((q, k, v, table, n), {"scale": float("inf")}, dps.DpsError), ((q, k[..., 8:], v[..., 8:], table, n), {}, ValueError)]:
        with pytest.raises(error):
            dps.dps_paged_attention(*args, **{"workspace": ws, **kw})
    assert dps.dps_launch_count() == launches
    # the native and the ctypes way say the same
    for kw in ({}, {"stream": torch.cuda.current_stream()}):
        check(dps.dps_paged_attention(q, k, v, table, n, workspace=ws, **kw), q, k, v, table, n)
    assert binding._native.paged_attention(q, k, v, table, n, None, None, ws) is not None
    assert ctypes.sizeof(binding.KvCache) == 64
