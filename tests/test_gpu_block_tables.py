"""GPU: a step's block tables, positions and slots, against the requests taken one after another."""
import numpy as np
import pytest
import torch

import paper_2609_34380_b200 as dps
from paper_2609_34380_b200 import binding
from tests import step_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def run(lengths, new, granted, table, page, blocks, tokens, native=True):
    dev = lambda a, t: torch.tensor(np.asarray(a), dtype=t, device=DEV)  # noqa: E731
    t = dev(table, torch.int32)
    B = len(lengths)
    filled = lambda n, dtype: torch.full((n,), 77, dtype=dtype, device=DEV)  # noqa: E731
    out = (filled(B, torch.int32), filled(B + 1, torch.int32), filled(tokens, torch.int32), filled(tokens, torch.int64), filled(1, torch.int32))
    g = dev(granted, torch.int32) if len(granted) else None
    got = dps.dps_extend_block_tables(dev(lengths, torch.int32), dev(new, torch.int32), g, t, page, blocks, *out,
                                      **({} if native else {"stream": torch.cuda.current_stream()}))
    return {**dict(zip(("lengths", "starts", "positions", "slots", "used"), (x.cpu().numpy() for x in got))), "table": t.cpu().numpy()}


def check(lengths, new, granted, table, page, blocks, tokens, native=True):
    want, bad = ref.extend_tables(lengths, new, granted, table, page, blocks, tokens)
    got = run(lengths, new, granted, table, page, blocks, tokens, native)
    status = dps.dps_stream_status()
    for name, value in want.items():
        assert np.array_equal(got[name], value), name
    assert status == (binding.DPS_ERR_DATA if bad else dps.DPS_OK)
    return bad


def problem(lengths, new, page, seed, spare=3, width=None):
    rng = np.random.default_rng(seed)
    have, need = [-(-n // page) for n in lengths], [-(-(n + m) // page) for n, m in zip(lengths, new)]
    blocks = sum(need) + spare + 1
    order = rng.permutation(blocks)
    table = np.full((len(lengths), width or max(need + [0]) + 2), -1, np.int64)
    at = 0
    for b, n in enumerate(have):
        table[b, :n] = order[at:at + n]
        at += n
    return lengths, new, order[at:at + sum(need) - sum(have) + spare], table, page, blocks


@pytest.mark.parametrize("page", [1, 7, 16, 128])
@pytest.mark.parametrize("native", [True, False])
def test_edges_of_blocks(page, native):
    lengths = [0, 0, 1, page - 1, page, page + 1, 5 * page, 5 * page - 1, 3]
    for new in ([1] * 9, [0] * 9, [0, 5 * page, 1, 1, 1, page, page - 1, 2 * page + 1, 0], [page] * 9):
        p = problem(lengths, new, page, 3)
        for pad in (0, 1, 40):
            assert not check(*p, sum(new) + pad, native=native)


@pytest.mark.parametrize("B", [1, 2, 31, 1023, 1024, 1025, 5000])
def test_many_requests(B):
    rng = np.random.default_rng(B)
    lengths = rng.integers(0, 300, B).tolist()
    for new in (np.ones(B, int).tolist(), rng.integers(0, 4, B).tolist(), (rng.random(B) < 0.01).astype(int).tolist()):
        assert not check(*problem(lengths, new, 16, B), sum(new) + 5)


def test_long_prompts():
    assert not check(*problem([0, 100, 7], [70001, 1, 9000], 16, 5), 80000)
    assert not check(*problem([1000000], [3], 128, 6), 3)


def test_nothing_to_do():
    assert not check([], [], [], np.zeros((0, 4), int), 16, 10, 5)
    assert not check(*problem([0, 0], [0, 0], 16, 7), 0)


def test_requests_that_are_left_out():
    p = problem([10, 20, 30, 40, 50], [20, 1, 40, 1, 3], 16, 8, spare=0)
    lengths, new, granted, table, page, blocks = p
    total = sum(new)
    assert check(lengths, new, granted[:-1], table, page, blocks, total)             # one block too few: the last that takes one
    assert check(lengths, new, granted[:1], table, page, blocks, total)              # the third does not get its share, the fourth needs none
    assert check(lengths, new, [], table, page, blocks, total)
    assert check(lengths, new, granted, table, page, blocks, total - 1)              # rows behind the end
    assert check(lengths, new, granted, table, page, blocks, 21)
    assert check(lengths, new, granted, table[:, :4], page, blocks, total)           # a table too narrow for the third
    for b, field, value in [(1, 0, -1), (1, 1, -1), (2, 1, 2 ** 31 - 1), (0, 0, 2 ** 31 - 1), (2, 1, -2 ** 31), (0, 0, -2 ** 31)]:
        changed = [list(lengths), list(new)]
        changed[field][b] = value
        assert check(*changed, granted, table, page, blocks, total)
    many = [[2 ** 31 - 1] * 4, [2 ** 31 - 1] * 4]                                    # sums beyond 32 bits
    got = run(*many, granted, table[:4], page, blocks, 8)
    assert dps.dps_stream_status() == binding.DPS_ERR_DATA
    assert (got["slots"] == -1).all() and (got["lengths"] == 2 ** 31 - 1).all() and got["used"][0] == 0 and got["starts"][-1] == 2 ** 31 - 1
    assert np.array_equal(got["table"], table[:4])


def test_bad_block_ids():
    lengths, new, granted, table, page, blocks = problem([10, 20, 30], [20, 1, 40], 16, 9)
    for bad in (-1, blocks, 2 ** 31 - 1, -2 ** 31):
        g, t = granted.copy(), table.copy()
        g[1] = bad
        assert check(lengths, new, g, table, page, blocks, sum(new))
        t[1, 1] = bad
        assert check(lengths, new, granted, t, page, blocks, sum(new))


def test_a_view_of_a_larger_table_and_default_outputs():
    lengths, new, granted, table, page, blocks = problem([10, 20, 30], [20, 1, 40], 16, 10)
    dev = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32, device=DEV)  # noqa: E731
    wide = torch.full((3, table.shape[1] + 6), 9, dtype=torch.int32, device=DEV)
    inside = wide[:, 2:-4]
    inside.copy_(dev(table))
    after, starts, positions, slots, used = dps.dps_extend_block_tables(dev(lengths), dev(new), dev(granted), inside, page, blocks, tokens=70)
    want, _ = ref.extend_tables(lengths, new, granted, table, page, blocks, 70)
    for got, name in ((after, "lengths"), (starts, "starts"), (positions, "positions"), (slots, "slots"), (used, "used"), (inside, "table")):
        assert np.array_equal(got.cpu().numpy(), want[name]), name
    assert bool((wide[:, :2] == 9).all()) and bool((wide[:, -4:] == 9).all())
    # slots beyond 2^31
    t = dev([[2 ** 31 - 2]])
    _, _, _, slots, _ = dps.dps_extend_block_tables(dev([5]), dev([2]), None, t, 64, 2 ** 31 - 1, tokens=2)
    assert slots.tolist() == [(2 ** 31 - 2) * 64 + 5, (2 ** 31 - 2) * 64 + 6]
    assert dps.dps_stream_status() == dps.DPS_OK


def test_captured_and_replayed():
    lengths, new, granted, table, page, blocks = problem([15, 16, 0], [1, 1, 1], 16, 11)
    dev = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32, device=DEV)  # noqa: E731
    n, m, g, t = dev(lengths), dev(new), dev(granted), dev(table)
    out = dps.dps_extend_block_tables(n, m, g, t, page, blocks, tokens=6)
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        dps.dps_extend_block_tables(n, m, g, t, page, blocks, *out)
    now = ([16, 16, 0], [1, 0, 3])
    n.copy_(dev(now[0])), m.copy_(dev(now[1])), t.copy_(dev(table))
    graph.replay()
    want, _ = ref.extend_tables(*now, granted, table, page, blocks, 6)
    for got, name in zip((*out, t), ("lengths", "starts", "positions", "slots", "used", "table")):
        assert np.array_equal(got.cpu().numpy(), want[name]), name
    assert dps.dps_stream_status() == dps.DPS_OK


def test_refusals():
    dev = lambda a, dtype=torch.int32: torch.tensor(a, dtype=dtype, device=DEV)  # noqa: E731
    n, m, t, g = dev([3, 4]), dev([1, 1]), dev([[0, 1], [2, 3]]), dev([4, 5])
    launches = dps.dps_launch_count()
    for args, kw, error in [
            ((n, m[:1], g, t, 16, 9), {"tokens": 2}, ValueError), ((n.long(), m, g, t, 16, 9), {"tokens": 2}, TypeError),
            ((n, m, g, t[:1], 16, 9), {"tokens": 2}, ValueError), ((n, m, g, t.long(), 16, 9), {"tokens": 2}, TypeError),
            ((n, m, g, t.t().contiguous().t(), 16, 9), {"tokens": 2}, ValueError), ((n, m, g, t, 0, 9), {"tokens": 2}, dps.DpsError),
            ((n, m, g, t, 16, 9), {}, ValueError), ((n, m, g, t, 16, 9, n), {"tokens": 2}, dps.DpsError),
            ((n, m, g, t, 16, 9), {"positions": dev([0, 0]), "tokens": 3}, ValueError),
            ((n, m, g, t, 16, 9), {"positions": dev([0, 0]), "slots": dev([0, 0])}, TypeError),
            ((n, m, g, t, 2 ** 32 + 16, 9), {"tokens": 2}, ValueError), ((n, m, g.cpu(), t, 16, 9), {"tokens": 2}, ValueError)]:
        with pytest.raises(error):
            dps.dps_extend_block_tables(*args, **kw)
    with pytest.raises(ValueError):                         # outputs given and another number of tokens
        dps.dps_extend_block_tables(n, m, g, t, 16, 9, dev([0, 0]), dev([0, 0, 0]), dev([0, 0]), dev([0, 0], torch.int64), dev([0]), tokens=3)
    assert dps.dps_launch_count() == launches
