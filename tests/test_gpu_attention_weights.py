"""GPU: paged attention where most of the answer comes from weights far below the largest one."""
import math

import pytest
import torch

import paper_2609_34380_b200 as dps
from tests import step_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
# What 16-bit weights hold of a weight: their two values have 11 (FP16) or 8 (BF16) bits each, so 2^-21 or 2^-15 of the weight is left out at most.
# FP16 ends at 2^-24; the weights are lifted by 2^15 before they are cut, so nothing finer than 2^-39 of the largest weight is held, half a step of it off.
RELATIVE = {torch.float16: 2.0 ** -21, torch.bfloat16: 2.0 ** -15}
ABSOLUTE = {torch.float16: 2.0 ** -40, torch.bfloat16: 0.0}


def problem(lengths, heads, kv_heads, dim, gap, sink, dtype, seed):
    """Keys whose scores are their first element; the sink's score is `gap` above the others' centre, and its value is zero.  `sink`: where it stands, as a
    share of the request's length."""
    k, v, table = ref.paged_cache(lengths, 16, kv_heads, dim, dtype, seed)
    g = torch.Generator().manual_seed(seed + 1)
    for b, n in enumerate(lengths):
        at = min(int(sink * n), n - 1)
        block, within = int(table[b, at // 16]), at % 16
        k[block, within, :, 0], v[block, within] = gap, 0.0
    used = torch.isfinite(v)
    v[used] = (v[used].float().abs() * 500 + 250 * (v[used] != 0)).to(dtype)             # one sign and far from zero: nothing cancels, no output is subnormal
    q = torch.zeros((len(lengths), heads, dim), dtype=dtype)
    q[..., 0] = (torch.rand((len(lengths), heads), generator=g) * 0.25 + 0.75).to(dtype)
    return q.to(DEV), k, v, table, torch.tensor(lengths, dtype=torch.int32, device=DEV)


def check(got, q, k, v, table, lengths, dtype):
    """A score is one product of two 16-bit numbers, exact in 32 bits.  Times scale_log2, minus the maximum, through the exponential: each rounds
    once, at a size of at most |s| / ln 2, and the exponential is off by 2^-22: d.  Sums of 32 bits as everywhere."""
    share = q.shape[1] // k.shape[2]
    for b, n in enumerate(lengths.tolist()):
        blocks = table[b, :-(-n // k.shape[1])].long()
        scores = q[b, :, :1].double() * k[blocks].flatten(0, 1)[:n, :, 0].double().t().repeat_interleave(share, 0)            # [heads][tokens]
        values = v[blocks].flatten(0, 1)[:n].double().repeat_interleave(share, 1)
        w = torch.softmax(scores, 1)
        want = torch.einsum("ht,thd->hd", w, values)
        d = 6 * ref.U32 * scores.abs().amax(1)[:, None] + 2.0 ** -22
        spread = torch.einsum("ht,thd->hd", w, values.abs())
        bound = ref.half_unit(dtype) * want.abs() + spread * (2 * d + RELATIVE[dtype] + (n / 16 + 64) * 4 * ref.U32) \
            + ABSOLUTE[dtype] * w.amax(1)[:, None] * values.abs().sum(0) + torch.finfo(dtype).smallest_normal * 2.0 ** -11
        off = (got[b].double() - want).abs()
        assert bool(torch.isfinite(got[b]).all())
        assert bool((off <= bound).all()), (b, float((off / bound).max()), float((off / want.abs()).max()))


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("gap", [4.0, 10.0, 14.0, 16.0, 17.5, 19.0, 21.0])
@pytest.mark.parametrize("lengths,heads,kv_heads,dim", [([8190, 4000, 17, 8190, 2049], 4, 4, 64), ([20000], 8, 1, 128), ([3000] * 41, 16, 8, 64), ([5000, 900], 12, 1, 128),
                                                        ([6000, 333], 2, 2, 256)])
def test_many_small_weights_beside_a_large_one(dtype, gap, lengths, heads, kv_heads, dim):
    for sink in (0.0, 0.37, 1.0):
        p = problem(lengths, heads, kv_heads, dim, gap, sink, dtype, 7)
        check(dps.dps_paged_attention(*p, scale=1.0), *p, dtype)
    assert dps.dps_stream_status() == dps.DPS_OK


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_equal_small_weights(dtype):
    """All scores but one are the same, so that every weight is cut the same way and the errors add up."""
    for gap in (13.0, 15.0, 16.6, 17.3, 18.0):
        q, k, v, table, n = problem([8190] * 8, 8, 8, 64, gap, 0.0, dtype, 9)
        q[..., 0] = 1.0
        first = table[:, 0].long()
        keep = k[first, 0].clone()
        k[torch.isfinite(k)] = 0.0
        k[first, 0] = keep
        check(dps.dps_paged_attention(q, k, v, table, n, scale=1.0), q, k, v, table, n, dtype)
        assert math.isclose(float(k[first[0], 0, 0, 0]), gap, rel_tol=0.01)
