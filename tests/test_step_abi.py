"""CPU: the C ABI of the operators between the linears rejects bad arguments before it touches a device."""
import ctypes
import subprocess
from pathlib import Path

import pytest
import torch

import paper_2609_34380_b200 as dps
from paper_2609_34380_b200 import binding

ROOT = Path(__file__).resolve().parents[1]
FAKE, ODD, HALF = (ctypes.c_void_p(p) for p in (0x10000, 0x10002, 0x10008))   # never dereferenced: every call below fails first


def far(i):
    return ctypes.c_void_p(0x1000000 * (i + 1))


def cache(**kw):
    c = dict(k=0x10000, v=0x20000, blocks=10, block_stride=16 * 2 * 64, token_stride=2 * 64, head_stride=64, page_tokens=16, heads=2, head_dim=64, type=0)
    return binding.KvCache(**{**c, **kw})


BAD_CACHES = [(dict(type=2), binding.DPS_ERR_UNSUPPORTED), (dict(head_dim=0), binding.DPS_ERR_SHAPE), (dict(head_dim=264), binding.DPS_ERR_SHAPE),
              (dict(head_dim=60), binding.DPS_ERR_SHAPE), (dict(heads=0), binding.DPS_ERR_SHAPE), (dict(page_tokens=0), binding.DPS_ERR_SHAPE),
              (dict(page_tokens=-16), binding.DPS_ERR_SHAPE), (dict(blocks=-1), binding.DPS_ERR_SHAPE), (dict(blocks=1 << 31), binding.DPS_ERR_SHAPE),
              (dict(token_stride=-128), binding.DPS_ERR_SHAPE), (dict(token_stride=132), binding.DPS_ERR_ALIGN), (dict(head_stride=4), binding.DPS_ERR_ALIGN),
              (dict(block_stride=2 ** 62), binding.DPS_ERR_SHAPE), (dict(k=0), binding.DPS_ERR_NULL), (dict(v=0), binding.DPS_ERR_NULL),
              (dict(k=0x10008), binding.DPS_ERR_ALIGN)]


def test_paged_attention():
    lib = binding.library()
    need = lib.dps_paged_attention_workspace_bytes(8, 2, 64)

    def call(c=None, q=FAKE, row=512, head=64, B=3, heads=8, table=FAKE, stride=20, width=20, lengths=FAKE, scale=0.1, out=FAKE, ws=FAKE, bytes_=need):
        c = cache() if c is None else c
        return lib.dps_paged_attention(q, row, head, B, heads, ctypes.byref(c), table, stride, width, lengths, scale, out, ws, bytes_, None)
    for kw, status in BAD_CACHES:
        assert call(cache(**kw)) == status, kw
    assert lib.dps_paged_attention(FAKE, 512, 64, 3, 8, None, FAKE, 20, 20, FAKE, 0.1, FAKE, FAKE, need, None) == binding.DPS_ERR_NULL
    for kw, status in [(dict(B=-1), "SHAPE"), (dict(B=(1 << 20) + 1), "SHAPE"), (dict(heads=0), "SHAPE"), (dict(heads=7), "SHAPE"), (dict(width=-1), "SHAPE"),
                       (dict(stride=19), "SHAPE"), (dict(width=1 << 31), "SHAPE"), (dict(row=-8), "SHAPE"), (dict(row=516), "ALIGN"), (dict(head=60), "ALIGN"),
                       (dict(row=2 ** 62), "SHAPE"), (dict(scale=float("nan")), "SHAPE"), (dict(scale=float("-inf")), "SHAPE"), (dict(q=None), "NULL"),
                       (dict(lengths=None), "NULL"), (dict(out=None), "NULL"), (dict(table=None), "NULL"), (dict(q=HALF), "ALIGN"), (dict(out=HALF), "ALIGN"),
                       (dict(table=ODD), "ALIGN"), (dict(lengths=ODD), "ALIGN"), (dict(ws=None), "WORKSPACE"), (dict(ws=HALF), "WORKSPACE"),
                       (dict(bytes_=need - 1), "WORKSPACE")]:
        assert call(**kw) == getattr(binding, "DPS_ERR_" + status), kw
    assert call(B=0, q=None, table=None, lengths=None, out=None, ws=None) == binding.DPS_OK
    bytes_of = lib.dps_paged_attention_workspace_bytes
    assert 0 < bytes_of(1, 1, 8) <= need <= bytes_of(8, 1, 128) <= bytes_of(16, 1, 128)
    for bad in [(0, 1, 64), (4, 0, 64), (4, 3, 64), (4, 2, 0), (4, 2, 260), (4, 2, 12), (-4, 2, 64)]:
        assert bytes_of(*bad) == 0
    assert lib.dps_paged_attention_workspace_init(None, need, None) == binding.DPS_ERR_WORKSPACE
    assert lib.dps_paged_attention_workspace_init(HALF, need, None) == binding.DPS_ERR_WORKSPACE
    assert lib.dps_paged_attention_workspace_init(FAKE, 64, None) == binding.DPS_ERR_WORKSPACE


def test_qk_norm_rope():
    lib = binding.library()

    def call(c=None, qkv=FAKE, stride=768, T=3, heads=8, slots=FAKE, pos=FAKE, table=FAKE, most=100, rotated=64, inter=0, qw=None, kw_=None, eps=1e-6,
             out=FAKE, out_stride=512):
        c = cache() if c is None else c
        return lib.dps_qk_norm_rope(qkv, stride, T, heads, ctypes.byref(c), slots, pos, table, most, rotated, inter, qw, kw_, eps, out, out_stride, None)
    for kw, status in BAD_CACHES:
        assert call(cache(**kw)) == status, kw
    for kw, status in [(dict(T=-1), "SHAPE"), (dict(T=1 << 31), "SHAPE"), (dict(heads=-1), "SHAPE"), (dict(rotated=8), "SHAPE"), (dict(rotated=80), "SHAPE"),
                       (dict(rotated=-16), "SHAPE"), (dict(most=-1), "SHAPE"), (dict(eps=-1.0), "SHAPE"), (dict(eps=float("nan")), "SHAPE"),
                       (dict(stride=760), "SHAPE"), (dict(stride=772), "ALIGN"), (dict(out_stride=504), "SHAPE"), (dict(out_stride=516), "ALIGN"),
                       (dict(stride=2 ** 61), "SHAPE"), (dict(qkv=None), "NULL"), (dict(slots=None), "NULL"), (dict(out=None), "NULL"), (dict(pos=None), "NULL"),
                       (dict(table=None), "NULL"), (dict(qw=FAKE), "NULL"), (dict(kw_=FAKE), "NULL"), (dict(qkv=HALF), "ALIGN"), (dict(out=HALF), "ALIGN"),
                       (dict(table=HALF), "ALIGN"), (dict(qw=HALF, kw_=FAKE), "ALIGN"), (dict(slots=ctypes.c_void_p(0x10004)), "ALIGN"), (dict(pos=ODD), "ALIGN"),
                       (dict(T=(1 << 31) - 1, heads=65535, stride=65539 * 64, out_stride=65535 * 64), "SHAPE")]:
        assert call(**kw) == getattr(binding, "DPS_ERR_" + status), kw
    # queries in place, but in rows of another stride: a warp would write what another one has yet to read
    assert call(qkv=FAKE, out=FAKE) == binding.DPS_ERR_DATA
    assert call(T=0, qkv=None, slots=None, out=None, pos=None, table=None) == binding.DPS_OK


def test_extend_block_tables():
    lib = binding.library()

    def call(lengths=far(0), new=far(1), B=4, granted=far(2), G=8, table=far(3), stride=10, width=10, page=16, blocks=100, after=far(4), starts=far(5),
             positions=far(6), slots=far(7), T=8, used=far(8)):
        return lib.dps_extend_block_tables(lengths, new, B, granted, G, table, stride, width, page, blocks, after, starts, positions, slots, T, used, None)
    for kw, status in [(dict(B=-1), "SHAPE"), (dict(B=(1 << 20) + 1), "SHAPE"), (dict(G=-1), "SHAPE"), (dict(G=1 << 31), "SHAPE"), (dict(T=-1), "SHAPE"),
                       (dict(T=1 << 31), "SHAPE"), (dict(page=0), "SHAPE"), (dict(width=-1), "SHAPE"), (dict(stride=9), "SHAPE"), (dict(blocks=-1), "SHAPE"),
                       (dict(blocks=1 << 31), "SHAPE"), (dict(stride=2 ** 61), "SHAPE"), (dict(lengths=None), "NULL"), (dict(new=None), "NULL"),
                       (dict(granted=None), "NULL"), (dict(table=None), "NULL"), (dict(after=None), "NULL"), (dict(starts=None), "NULL"),
                       (dict(positions=None), "NULL"), (dict(slots=None), "NULL"), (dict(used=None), "NULL"), (dict(lengths=ODD), "ALIGN"),
                       (dict(slots=ctypes.c_void_p(0x10004)), "ALIGN"), (dict(after=far(0)), "DATA"), (dict(after=far(1)), "DATA"),
                       (dict(after=ctypes.c_void_p(0x1000000 + 12)), "DATA")]:
        assert call(**kw) == getattr(binding, "DPS_ERR_" + status), kw


def test_route_experts():
    lib = binding.library()

    def call(logits=FAKE, stride=64, type_=0, T=4, E=64, bias=None, scoring=0, groups=1, top_groups=1, top=2, renorm=1, scale=1.0, token=None, expert=FAKE, w=FAKE):
        return lib.dps_route_experts(logits, stride, type_, T, E, bias, scoring, groups, top_groups, top, renorm, scale, token, expert, w, None)
    for kw, status in [(dict(type_=3), "UNSUPPORTED"), (dict(type_=-1), "UNSUPPORTED"), (dict(scoring=2), "MODE"), (dict(T=-1), "SHAPE"), (dict(E=0), "SHAPE"),
                       (dict(E=1025, stride=1025), "SHAPE"), (dict(groups=0), "SHAPE"), (dict(groups=5), "SHAPE"), (dict(groups=64), "SHAPE"),
                       (dict(top_groups=0), "SHAPE"), (dict(top_groups=2), "SHAPE"), (dict(top=0), "SHAPE"), (dict(top=33), "SHAPE"),
                       (dict(groups=16, top_groups=2, top=9), "SHAPE"), (dict(stride=63), "SHAPE"), (dict(T=1 << 30, top=2), "SHAPE"), (dict(logits=None), "NULL"),
                       (dict(expert=None), "NULL"), (dict(w=None), "NULL"), (dict(logits=ODD, type_=2), "ALIGN"), (dict(bias=ODD), "ALIGN"),
                       (dict(token=ODD), "ALIGN"), (dict(expert=ODD), "ALIGN"), (dict(w=ODD), "ALIGN")]:
        assert call(**kw) == getattr(binding, "DPS_ERR_" + status), kw
    assert call(T=0, logits=None, expert=None, w=None) == binding.DPS_OK


def test_host_tensors_are_refused():
    h, i = torch.zeros((2, 8, 64), dtype=torch.float16), torch.zeros(2, dtype=torch.int32)
    c, t = torch.zeros((3, 16, 2, 64), dtype=torch.float16), torch.zeros((2, 3), dtype=torch.int32)
    with pytest.raises(ValueError):
        dps.dps_paged_attention(h, c, c, t, i)
    with pytest.raises(ValueError):
        dps.dps_qk_norm_rope(torch.zeros((2, 768), dtype=torch.float16), c, c, torch.zeros(2, dtype=torch.int64))
    with pytest.raises(ValueError):
        dps.dps_extend_block_tables(i, i, None, t, 16, 3, tokens=2)
    with pytest.raises(ValueError):
        dps.dps_route_experts(torch.zeros((2, 8)), 2)
    with pytest.raises(ValueError):
        binding._int32(1 << 31, "page_tokens")
    native = binding._native
    if native is not None:                                  # what the native entries do not take goes the other way
        assert native.paged_attention(h, c, c, t, i, None, None, None) is None and native.paged_attention() is None
        assert native.qk_norm_rope(1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11) is None and native.extend_block_tables(*[None] * 11) is None
        assert native.route_experts(h, 2, None, 0, 1, 1, True, 1.0, None, None, None) is None


def test_the_struct_is_the_headers(tmp_path):
    """Offsets and size as a C compiler lays them out."""
    names = [f for f, _ in binding.KvCache._fields_]
    (tmp_path / "t.c").write_text('#include <stdio.h>\n#include "dps.h"\nint main(void) {' + "".join(
        f'printf("%zu ", offsetof(dps_kv_cache, {n}));' for n in names) + 'printf("%zu", sizeof(dps_kv_cache)); return 0; }')
    subprocess.run(["gcc", "-I", str(ROOT / "include"), str(tmp_path / "t.c"), "-o", str(tmp_path / "t")], check=True)
    out = subprocess.run([str(tmp_path / "t")], capture_output=True, text=True, check=True).stdout.split()
    assert [int(x) for x in out] == [getattr(binding.KvCache, n).offset for n in names] + [ctypes.sizeof(binding.KvCache)]
