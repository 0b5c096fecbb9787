"""GPU: infinities and NaN among the values that paged attention sums."""
import pytest
import torch

import paper_2609_34380_b200 as dps
from tests import step_reference as ref

pytestmark = pytest.mark.gpu
DEV, INF, NAN = "cuda:0", float("inf"), float("nan")


def problem(lengths, heads, kv_heads, dim, page, dtype, seed):
    k, v, table = ref.paged_cache(lengths, page, kv_heads, dim, dtype, seed)
    g = torch.Generator().manual_seed(seed + 1)
    q = torch.randn((len(lengths), heads, dim), generator=g).to(dtype).to(DEV)
    return q, k, v, table, torch.tensor(lengths, dtype=torch.int32, device=DEV)


def put(v, table, b, t, h, d, value):
    v[int(table[b, t // v.shape[1]]), t % v.shape[1], h, d] = value


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("lengths,heads,kv_heads,dim,page", [([1, 0, 40, 300], 4, 4, 64, 16), ([20011, 5], 8, 1, 128, 16), ([700, 64, 9000], 12, 1, 96, 24),
                                                             ([3000, 90], 20, 1, 128, 16), ([2500, 33], 4, 2, 256, 7), ([90, 500], 6, 2, 40, 1)])
def test_an_infinite_element_gives_that_infinity(dtype, lengths, heads, kv_heads, dim, page):
    """One token's infinity at a time, at every kind of place, whatever its weight: sum p_t V_t is that infinity, and the other elements are as they were."""
    q, k, v, table, n = problem(lengths, heads, kv_heads, dim, page, dtype, 3)
    ws = dps.dps_paged_attention_workspace(heads, kv_heads, dim)
    plain = dps.dps_paged_attention(q, k, v, table, n, workspace=ws)
    share = heads // kv_heads
    for b, length in enumerate(lengths):
        for t in sorted({0, length // 3, length // 2, length - 1}) if length else []:
            for sign in (INF, -INF):
                bad, want = v.clone(), plain.clone()
                h, d = (t + b) % kv_heads, (5 * t + 3) % dim
                put(bad, table, b, t, h, d, sign)
                put(bad, table, b, length - 1, h, (d + 4) % dim, sign)
                want[b, h * share:(h + 1) * share, d] = sign
                want[b, h * share:(h + 1) * share, (d + 4) % dim] = sign
                got = dps.dps_paged_attention(q, k, bad, table, n, workspace=ws)
                assert torch.equal(got, want), (b, t, sign)
    assert dps.dps_stream_status() == dps.DPS_OK


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("lengths,heads,kv_heads,dim", [([50], 1, 1, 64), ([20011], 8, 2, 128), ([400, 3], 12, 1, 128), ([1200], 2, 1, 256)])
def test_infinities_that_meet(dtype, lengths, heads, kv_heads, dim):
    q, k, v, table, n = problem(lengths, heads, kv_heads, dim, 16, dtype, 5)
    share, last = heads // kv_heads, lengths[0] - 1
    want = dps.dps_paged_attention(q, k, v, table, n)
    for d, (first, second, result) in enumerate([(INF, INF, INF), (-INF, -INF, -INF), (INF, -INF, NAN), (NAN, 1.0, NAN), (NAN, INF, NAN), (0.0, 0.0, None)]):
        put(v, table, 0, 1, 0, d, first), put(v, table, 0, last, 0, d, second)
        if result is not None:
            want[0, :share, d] = result
    got = dps.dps_paged_attention(q, k, v, table, n)
    want[0, :share, 5] = got[0, :share, 5]
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got.nan_to_num(nan=7.0), want.nan_to_num(nan=7.0))


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_infinities_of_small_weights_and_behind_the_length(dtype):
    """Weights down to nothing that 32 bits hold, an infinity that the running sums are rescaled over, and infinities of tokens that do not count."""
    q, k, v, table, n = problem([600, 80], 8, 2, 64, 16, dtype, 11)
    k[torch.isfinite(k)] = 0.0
    q[..., 0] = 1.0
    put(k, table, 0, 300, slice(None), 0, 1000.0)                            # a score of 125: every other weight is e^-125
    plain = dps.dps_paged_attention(q, k, v, table, n)
    for t in (0, 299, 301, 599):
        bad, want = v.clone(), plain.clone()
        put(bad, table, 0, t, 1, 9, -INF)
        want[0, 4:, 9] = -INF
        assert torch.equal(dps.dps_paged_attention(q, k, bad, table, n), want), t
    bad = v.clone()
    bad[~torch.isfinite(bad)] = INF                                         # behind the lengths, and blocks of nobody
    assert torch.equal(dps.dps_paged_attention(q, k, bad, table, n), plain)
    # without a softmax there is no answer, infinite values or not
    put(k, table, 1, 5, slice(None), 0, INF)
    put(bad, table, 1, 9, 0, 3, INF)
    assert bool(torch.isnan(dps.dps_paged_attention(q, k, bad, table, n)[1]).all())
    assert dps.dps_stream_status() == dps.DPS_OK


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("lengths,heads,kv_heads,dim", [([40, 9], 2, 2, 64), ([30000, 70], 16, 1, 128)])
def test_scores_of_minus_infinity(dtype, lengths, heads, kv_heads, dim):
    """A token whose score is -Inf has no weight; its value counts only if it is infinite.  If all scores are -Inf there is no answer."""
    q, k, v, table, n = problem(lengths, heads, kv_heads, dim, 16, dtype, 17)
    q = q.abs() + 0.25
    for t in (0, 5, lengths[0] // 2, lengths[0] - 1):
        put(k, table, 0, t, slice(None), slice(None), -INF)
    want = dps.dps_paged_attention(q, k, v, table, n)
    assert bool(torch.isfinite(want).all())
    put(v, table, 0, lengths[0] // 2, 0, 7, INF), put(v, table, 0, 5, 0, 1, -INF)
    want[0, :heads // kv_heads, 7], want[0, :heads // kv_heads, 1] = INF, -INF
    assert torch.equal(dps.dps_paged_attention(q, k, v, table, n), want)
    k[torch.isfinite(k)] = -INF
    assert bool(torch.isnan(dps.dps_paged_attention(q, k, v, table, n)).all())
    assert dps.dps_stream_status() == dps.DPS_OK
