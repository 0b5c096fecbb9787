"""GPU: routing with more tokens than warps are resident, so that a warp goes on from one row to another, and saturated scores."""
import numpy as np
import pytest
import torch

import paper_2609_34380_b200 as dps
from paper_2609_34380_b200 import binding
from tests import step_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
WEIGHT_BOUND = 64 * ref.U32     # as for the single turns: a rounding of each score, of their sum and of two quotients or products


def choose(logits, top_k, bias, sigmoid, groups, top_groups):
    """All rows at once, in 64 bits; a stable sort keeps the lower index in front."""
    x = logits.double()
    s = 1 / (1 + torch.exp(-x)) if sigmoid else torch.softmax(x, 1)
    c = s if bias is None else s + bias.double()
    if top_groups < groups:
        g = c.view(len(x), groups, -1)
        worth = g.topk(min(2, g.shape[2]), 2)[0].sum(2)
        kept = torch.zeros_like(worth, dtype=torch.bool).scatter_(1, torch.sort(worth, dim=1, descending=True, stable=True)[1][:, :top_groups], True)
        c = torch.where(kept[:, :, None], g, -torch.inf).view(len(x), -1)
    expert = torch.sort(c, dim=1, descending=True, stable=True)[1][:, :top_k]
    w = s.gather(1, expert)
    return expert, w / w.sum(1, keepdim=True)


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
@pytest.mark.parametrize("T", [4735, 4736, 4737, 10007])
@pytest.mark.parametrize("E,top_k,groups,top_groups,sigmoid,biased", [(256, 8, 8, 4, True, True), (256, 8, 8, 4, False, True), (128, 8, 1, 1, False, False),
                                                                      (72, 6, 8, 3, True, True), (8, 2, 1, 1, False, False)])
def test_more_tokens_than_resident_warps(dtype, T, E, top_k, groups, top_groups, sigmoid, biased):
    """Rows that need 64 bits, and rows without a choice, in front of, between and behind ordinary ones of the same warp."""
    g = torch.Generator().manual_seed(T + E)
    logits = torch.randn((T, E), generator=g).to(dtype)
    bias = (0.1 * torch.randn((E,), generator=g)).to(DEV) if biased else None
    near = torch.randperm(T, generator=g)[:T // 5]
    logits[near, 1] = logits[near, 0]                       # equal ones: a gap that 32 bits cannot judge
    off = torch.randperm(T, generator=g)[:T // 7]
    logits[off, E // 2] = float("-inf")
    logits = logits.to(DEV)
    bad = torch.randperm(T, generator=g)[:T // 11].to(DEV)
    logits[bad, E - 1] = float("nan")
    logits[T - 1, 0] = float("nan")
    token, expert, weights = dps.dps_route_experts(logits, top_k, bias, int(sigmoid), groups, top_groups)
    assert dps.dps_stream_status() == binding.DPS_ERR_DATA and dps.dps_stream_status() == dps.DPS_OK
    assert torch.equal(token, torch.arange(T, dtype=torch.int32, device=DEV).repeat_interleave(top_k))
    lost = torch.isnan(logits).any(1)
    expert = expert.view(T, top_k)
    assert bool((expert[lost] == -1).all()) and not bool(weights[lost].any())
    want, w = choose(logits[~lost], top_k, bias, sigmoid, groups, top_groups)
    assert torch.equal(expert[~lost].long(), want)
    assert bool(((weights[~lost].double() - w).abs() <= WEIGHT_BOUND * w.abs() + 1e-37).all())


def test_saturated_scores_are_equal():
    """Scores that 64 bits cannot tell apart are a tie, which falls on the lower index, with a bias or without one."""
    for bias in (None, torch.zeros(4, device=DEV)):
        for row, sigmoid, want in (([38.0, 0.0, 45.0, 50.0], 1, [0, 2]), ([0.0, -900.0, -800.0, -1000.0], 0, [0, 1])):
            _, expert, weights = dps.dps_route_experts(torch.tensor([row], device=DEV), 2, bias, sigmoid)
            experts, w = ref.route([row], 2, None if bias is None else np.zeros(4), bool(sigmoid), 1, 1, True, 1.0)
            assert expert.tolist() == want == experts[0].tolist() and np.allclose(weights.cpu().numpy(), w, atol=2.0 ** -22)
