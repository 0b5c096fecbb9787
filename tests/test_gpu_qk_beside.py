"""GPU: queries written beside the QKV rows that they come from."""
import pytest
import torch

import paper_2609_34380_b200 as dps
from paper_2609_34380_b200 import binding
from tests.test_gpu_qk_norm_rope import check, problem

pytestmark = pytest.mark.gpu


def test_columns_of_one_buffer():
    heads, kv_heads, dim = 8, 2, 64
    for T in (1, 19):
        for before in (True, False):                        # the queries' columns in front of qkv's, or behind them
            p = list(problem(T, heads, kv_heads, dim, 8, torch.float16, 64, True, 8))
            dense, wide = p[0].clone(), torch.zeros((T, 20 * dim), dtype=torch.float16, device="cuda:0")
            p[0] = wide[:, 8 * dim:] if before else wide[:, :12 * dim]
            p[0].copy_(dense)
            q = (wide[:, :8 * dim] if before else wide[:, 12 * dim:]).unflatten(1, (heads, dim))
            dps.dps_qk_norm_rope(*p, q_out=q)
            check([dense, *p[1:]], q, heads, kv_heads, dim, 1e-6, False)
            assert torch.equal(p[0], dense)
            over = wide[:, 4 * dim:12 * dim].unflatten(1, (heads, dim))
            with pytest.raises(dps.DpsError) as caught:
                dps.dps_qk_norm_rope(*p, q_out=over)
            assert caught.value.status == binding.DPS_ERR_DATA
    assert dps.dps_stream_status() == dps.DPS_OK
