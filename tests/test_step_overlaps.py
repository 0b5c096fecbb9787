"""CPU: outputs that lie over inputs or over one another are refused before anything is launched."""
import ctypes

import pytest

from paper_2609_34380_b200 import binding

FIRST = 0x10000000


@pytest.mark.parametrize("out,other", [(o, i) for o in ("after", "starts", "positions", "slots", "used") for i in ("lengths", "new", "granted", "after", "starts", "positions", "slots", "used")
                                       if o != i])
def test_extend_block_tables(out, other):
    """Every output over every other array, by all of it and by its first or last element."""
    B, G, T = 4, 8, 8
    size = dict(lengths=4 * B, new=4 * B, granted=4 * G, after=4 * B, starts=4 * (B + 1), positions=4 * T, slots=8 * T, used=4, table=4 * B * 10)
    at = {name: FIRST + 0x100000 * i for i, name in enumerate(size)}
    for place in (at[other], at[other] + size[other] - 4 if out != "slots" else at[other] + size[other] - 8, at[other] - size[out] + 8):
        where = {k: ctypes.c_void_p(v) for k, v in {**at, out: place // 8 * 8 if out == "slots" else place}.items()}
        if where[out].value + size[out] <= at[other] or where[out].value >= at[other] + size[other]:
            continue
        st = binding.library().dps_extend_block_tables(where["lengths"], where["new"], B, where["granted"], G, where["table"], 10, 10, 16, 100, where["after"],
                                                       where["starts"], where["positions"], where["slots"], T, where["used"], None)
        assert st == binding.DPS_ERR_DATA, (out, other, place - at[other])


@pytest.mark.parametrize("column", [8, 64, 512, 576, 768 - 8, -8, -504, 2 * 768 + 8])
@pytest.mark.parametrize("T", [1, 3])
def test_queries_over_other_columns(T, column):
    """Eight query heads and two of keys and values, 64 elements each: queries written over anything but themselves."""
    if T == 1 and column > 768:
        return
    c = binding.KvCache(k=0x10000, v=0x20000, blocks=10, block_stride=16 * 2 * 64, token_stride=2 * 64, head_stride=64, page_tokens=16, heads=2, head_dim=64, type=0)
    fake = [ctypes.c_void_p(0x40000 * (i + 1)) for i in range(3)]

    def call(stride, out_stride, at=column):
        return binding.library().dps_qk_norm_rope(ctypes.c_void_p(FIRST), stride, T, 8, ctypes.byref(c), fake[0], fake[1], fake[2], 100, 64, 0, None, None, 1e-6,
                                                  ctypes.c_void_p(FIRST + 2 * at), out_stride, None)
    assert call(768, 768) == binding.DPS_ERR_DATA
    assert call(768, 512) == binding.DPS_ERR_DATA
    if T > 1:                                               # rows with room between them, too little for the queries
        assert call(1272, 1272, 768) == binding.DPS_ERR_DATA and call(1272, 1272, 768 - 1272) == binding.DPS_ERR_DATA


@pytest.mark.parametrize("B,row,head,at", [(3, 512, 64, 64), (3, 512, 64, -8), (3, 512, 64, 1528), (3, 768, 64, 0), (1, 512, 128, 0), (3, 64, 192, 0), (3, 768, 64, 512),
                                           (3, 4096, 64, 504), (3, 4096, 64, 2568), (3, 4096, 64, 4096 - 1528)])
def test_results_over_queries(B, row, head, at):
    """Eight heads of 64 elements: results over queries, unless they are dense and the same."""
    lib = binding.library()
    c = binding.KvCache(k=0x10000, v=0x20000, blocks=10, block_stride=16 * 2 * 64, token_stride=2 * 64, head_stride=64, page_tokens=16, heads=2, head_dim=64, type=0)
    fake = ctypes.c_void_p(0x40000)
    assert lib.dps_paged_attention(ctypes.c_void_p(FIRST), row, head, B, 8, ctypes.byref(c), fake, 20, 20, fake, 0.1, ctypes.c_void_p(FIRST + 2 * at), fake,
                                   lib.dps_paged_attention_workspace_bytes(8, 2, 64), None) == binding.DPS_ERR_DATA


@pytest.mark.parametrize("out", ["token", "expert", "weights"])
@pytest.mark.parametrize("type_,stride,at", [(0, 64, 0), (0, 64, 4 * 64 * 2 - 4), (0, 64, -60), (2, 64, 1000), (1, 200, 120), (1, 200, 340), (0, 64, "bias"), (2, 200, "bias")])
def test_choices_over_logits(out, type_, stride, at):
    """Four tokens of 64 experts, four choices each (64 bytes): outputs over the logits, by their first or last bytes too, or over the bias."""
    far = {"logits": FIRST, "bias": FIRST + 0x100000, "token": FIRST + 0x200000, "expert": FIRST + 0x300000, "weights": FIRST + 0x400000}
    far[out] = far["bias"] + 252 if at == "bias" else FIRST + at
    p = {k: ctypes.c_void_p(v) for k, v in far.items()}
    assert binding.library().dps_route_experts(p["logits"], stride, type_, 4, 64, p["bias"], 0, 1, 1, 4, 1, 1.0, p["token"], p["expert"], p["weights"],
                                               None) == binding.DPS_ERR_DATA
