"""GPU: experts of each token and their weights, against the definition in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2609_34380_b200 as dps
from paper_2609_34380_b200 import binding
from tests import step_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
# 32-bit weights: a rounding of each score, of their sum and of two quotients or products, and an exponential of up to 1024 summed terms
WEIGHT_BOUND = 64 * ref.U32


def check(logits, top_k, bias=None, sigmoid=False, groups=1, top_groups=1, renormalise=True, scale=1.0):
    got = dps.dps_route_experts(logits, top_k, bias, int(sigmoid), groups, top_groups, renormalise, scale)
    token, expert, weights = (x.cpu().numpy() for x in got)
    experts, want = ref.route(logits.double().cpu().numpy(), top_k, None if bias is None else bias.double().cpu().numpy(), sigmoid, groups, top_groups,
                              renormalise, scale)
    T = logits.shape[0]
    assert np.array_equal(token, np.repeat(np.arange(T), top_k))
    assert np.array_equal(expert.reshape(T, top_k), experts)
    assert np.all(np.abs(weights - want) <= WEIGHT_BOUND * np.abs(want) + 1e-37)
    return got


def draw(T, E, dtype, seed, spread=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((T, E), generator=g) * spread).to(dtype).to(DEV), (0.1 * torch.randn((E,), generator=g)).to(DEV)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("E,top_k,groups,top_groups", [
    (8, 2, 1, 1), (1, 1, 1, 1), (7, 7, 1, 1), (33, 5, 1, 1), (64, 6, 8, 3), (100, 8, 10, 4), (160, 6, 8, 3), (256, 8, 8, 4), (257, 8, 1, 1), (512, 32, 32, 7),
    (1000, 16, 5, 2), (1024, 10, 1, 1), (12, 3, 12, 3), (66, 4, 2, 1), (96, 24, 4, 3), (128, 8, 8, 8)])
def test_against_the_definition(dtype, sigmoid, E, top_k, groups, top_groups):
    logits, bias = draw(37, E, dtype, E + top_k)
    for b in (None, bias):
        for renormalise, scale in ((True, 1.0), (False, 2.5)):
            check(logits, top_k, b, sigmoid, groups, top_groups, renormalise, scale)
    assert dps.dps_stream_status() == dps.DPS_OK


@pytest.mark.parametrize("T", [1, 2, 3, 5, 1023])
def test_token_counts(T):
    logits, bias = draw(T, 64, torch.float16, T)
    check(logits, 6, bias, True, 8, 3)
    check(logits, 2)


def test_ties_fall_on_the_lower_index():
    for groups, top_groups in ((1, 1), (8, 4)):
        for sigmoid in (False, True):
            zero = torch.zeros((3, 64), dtype=torch.float16, device=DEV)
            check(zero, 8, None, sigmoid, groups, top_groups)
            few = torch.randint(0, 3, (50, 64), generator=torch.Generator().manual_seed(4)).to(torch.float16).to(DEV)
            check(few, 8, None, sigmoid, groups, top_groups)
            check(few, 8, torch.zeros(64, device=DEV), sigmoid, groups, top_groups)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("E", [8, 32, 64, 256])
def test_the_two_zeros_are_equal(dtype, E):
    """A row of zeros of either sign: the first experts, whatever the signs."""
    logits = torch.zeros((64, E), dtype=dtype, device=DEV)
    logits[torch.rand((64, E), device=DEV) < 0.5] = -0.0
    for kw in ({}, {"scoring": dps.DPS_SCORE_SIGMOID}, {"renormalise": False}, {"bias": torch.zeros(E, device=DEV)}):
        _, experts, weights = dps.dps_route_experts(logits, 4, **kw)
        assert torch.equal(experts.view(64, 4), torch.arange(4, dtype=torch.int32, device=DEV).expand(64, 4)), kw
        assert torch.equal(weights, weights[:1, :1].expand(64, 4)), kw


def test_choices_that_32_bits_cannot_tell_apart():
    """Scores that differ in the 9th digit: the sum with the bias decides in 64 bits."""
    rng = np.random.default_rng(5)
    x = rng.normal(0, 1, (200, 64))
    bias = np.zeros(64, np.float32)
    s = lambda v: 1 / (1 + np.exp(-v))  # noqa: E731
    logits = x.astype(np.float32)
    target = rng.uniform(0.9, 1.0, 64)
    bias = (target - s(logits[0].astype(np.float64))).astype(np.float32)      # row 0: all choices near their target
    logits[:, 1::2] = logits[:, ::2]
    bias[1::2] = bias[::2]
    for step in (1, -1):
        near = bias.copy()
        near[1::2] = np.nextafter(near[::2], np.float32(step * 9))            # a unit more, or less, than their neighbour
        check(torch.tensor(logits, device=DEV), 16, torch.tensor(near, device=DEV), True)
        check(torch.tensor(logits, device=DEV), 16, torch.tensor(near, device=DEV), False)
        check(torch.tensor(logits, device=DEV), 8, torch.tensor(near, device=DEV), True, 8, 4)
    # neighbouring logits on the flat end of the sigmoid, and far down the softmax
    for centre in (12.0, -12.0, 0.0, 80.0):
        row = np.full((8, 64), centre, np.float32)
        for i in range(64):
            row[:, i] = np.nextafter(row[:, i - 1], np.float32(np.inf)) if i else row[:, 0]
        row = np.ascontiguousarray(row[:, rng.permutation(64)])
        for sigmoid in (True, False):
            check(torch.tensor(row, device=DEV), 16, torch.zeros(64, device=DEV), sigmoid)
            check(torch.tensor(row, device=DEV), 16, None, sigmoid)


def test_extreme_logits():
    logits, bias = draw(20, 64, torch.float32, 6, spread=40.0)
    check(logits, 8), check(logits, 8, bias, True), check(logits, 8, bias, False, 8, 4)
    logits[:, 5] = float("-inf")                                              # an expert that is switched off
    logits[3, 7:] = float("-inf")
    check(logits, 8), check(logits, 8, None, True), check(logits, 32, bias, True)
    off = bias.clone()
    off[9] = float("-inf")
    check(logits, 32, off, True)
    check(logits.clamp(min=-1e4), 8, off, False, 8, 4)
    big = torch.full((2, 64), 3e38, device=DEV)
    check(big, 4), check(-big, 4), check(big, 4, None, True)
    gone = torch.full((1, 64), -1e5, device=DEV)                              # scores of zero: weights of zero
    check(gone, 4, None, True)
    assert dps.dps_stream_status() == dps.DPS_OK


def test_rows_without_a_choice():
    logits, bias = draw(6, 64, torch.float32, 7)
    _, expert0, weights0 = check(logits, 8, bias, False, 8, 4)
    for sigmoid, row in ((False, float("nan")), (True, float("nan")), (False, float("inf"))):
        bad = logits.clone()
        bad[2, 63] = row
        token, expert, weights = dps.dps_route_experts(bad, 8, bias, int(sigmoid), 8, 4)
        assert dps.dps_stream_status() == binding.DPS_ERR_DATA and dps.dps_stream_status() == dps.DPS_OK
        assert bool((expert.view(6, 8)[2] == -1).all()) and not bool(weights[2].any()) and token[16:24].tolist() == [2] * 8
        others = [0, 1, 3, 4, 5]
        if not sigmoid:
            assert torch.equal(expert.view(6, 8)[others], expert0.view(6, 8)[others]) and torch.equal(weights[others], weights0[others])
    all_off = torch.full((1, 64), float("-inf"), device=DEV)
    _, expert, _ = dps.dps_route_experts(all_off, 2)
    assert expert.tolist() == [-1, -1] and dps.dps_stream_status() == binding.DPS_ERR_DATA
    mixed = torch.zeros(64, device=DEV)                                       # a group that holds +Inf and -Inf is worth nothing that can be compared
    mixed[:8] = float("-inf")
    mixed[0] = float("inf")
    _, expert, _ = dps.dps_route_experts(logits, 8, mixed, 1, 8, 4)
    assert bool((expert == -1).all()) and dps.dps_stream_status() == binding.DPS_ERR_DATA


def test_strides_streams_and_graphs():
    wide = torch.full((11, 100), float("nan"), dtype=torch.bfloat16, device=DEV)
    logits, bias = draw(11, 64, torch.bfloat16, 8)
    wide[:, 7:71] = logits
    got = check(wide[:, 7:71], 6, bias, True, 8, 4)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        again = dps.dps_route_experts(wide[:, 7:71], 6, bias, 1, 8, 4, token_of_row=torch.empty_like(got[0]), expert_of_row=torch.empty_like(got[1]),
                                      weights=torch.empty_like(got[2]))
    wide[:, 7:71] = logits.flip(0)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(again[1].view(11, 6), got[1].view(11, 6).flip(0)) and torch.equal(again[2], got[2].flip(0))
    named = dps.dps_route_experts(logits, 6, bias, 1, 8, 4, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(named, got))
    assert dps.dps_route_experts(logits[:0], 6)[2].shape == (0, 6)


def test_refusals():
    logits, bias = draw(4, 64, torch.float16, 9)
    launches = dps.dps_launch_count()
    for args, kw, error in [
            ((logits.double(), 2), {}, TypeError), ((logits[0], 2), {}, ValueError), ((logits.t().contiguous().t(), 2), {}, ValueError),
            ((logits, 0), {}, dps.DpsError), ((logits, 33), {}, dps.DpsError), ((logits, -1), {}, dps.DpsError), ((logits, 65), {}, dps.DpsError),
            ((logits, 2, bias[:3]), {}, ValueError), ((logits, 2, bias.half()), {}, TypeError), ((logits, 2, bias, 2), {}, dps.DpsError),
            ((logits, 2, bias, 0, 5, 1), {}, dps.DpsError), ((logits, 2, bias, 0, 8, 9), {}, dps.DpsError), ((logits, 9, bias, 0, 8, 1), {}, dps.DpsError),
            ((logits, 2), {"weights": torch.empty(7, device=DEV)}, ValueError), ((logits, 2), {"expert_of_row": torch.empty(8, dtype=torch.int64, device=DEV)}, TypeError),
            ((logits, 2 ** 32 + 2), {}, ValueError)]:
        with pytest.raises(error):
            dps.dps_route_experts(*args, **kw)
    assert dps.dps_launch_count() == launches
    assert binding._native.route_experts(logits, 2, None, 0, 1, 1, True, 1.0, None, None, None) is not None
