"""GPU: paged attention whose results lie over the queries, or in the room between them."""
import pytest
import torch

import paper_2609_34380_b200 as dps
from paper_2609_34380_b200 import binding
from tests import step_reference as ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("lengths,heads,kv_heads,dim", [([20011], 8, 1, 128), ([1, 0, 700, 64], 40, 2, 64), ([5000, 33, 2], 24, 1, 256), ([300] * 90, 12, 4, 80)])
def test_results_in_place(dtype, lengths, heads, kv_heads, dim):
    k, v, table = ref.paged_cache(lengths, 16, kv_heads, dim, dtype, 3)
    B, n = len(lengths), torch.tensor(lengths, dtype=torch.int32, device="cuda:0")
    ws = dps.dps_paged_attention_workspace(heads, kv_heads, dim)
    for seed in range(5):
        q = torch.randn((B, heads, dim), generator=torch.Generator().manual_seed(seed)).to(dtype).to("cuda:0")
        want = dps.dps_paged_attention(q, k, v, table, n, workspace=ws)
        wide = torch.zeros((B, (heads * dim) * (1 + B)), dtype=dtype, device="cuda:0")     # rows of queries with room for all results between two of them
        between = wide[:, :heads * dim].unflatten(1, (heads, dim))
        between.copy_(q)
        room = wide.flatten()[heads * dim:heads * dim * (1 + B)].view(B, heads, dim)
        assert torch.equal(dps.dps_paged_attention(between, k, v, table, n, out=room, workspace=ws), want) and torch.equal(between, q)
        with pytest.raises(dps.DpsError) as caught:
            dps.dps_paged_attention(between, k, v, table, n, out=wide.flatten()[8:8 + heads * dim * B].view(B, heads, dim), workspace=ws)
        assert caught.value.status == binding.DPS_ERR_DATA
        got = dps.dps_paged_attention(q, k, v, table, n, out=q, workspace=ws)
        assert got is q and torch.equal(q, want)
    assert dps.dps_stream_status() == dps.DPS_OK
