"""What the 8-bit cache, its attention and the block tables refuse on the host, before anything is enqueued, and the plain
64-bit forms that their GPU tests use.  No GPU is touched."""
import ctypes as C
import os

import numpy as np
import pytest

from paper_2512_07993_amd import binding as B

from quant_helpers import VALUES, Pool, encode, scale_byte


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not os.path.exists(B._LIB_PATH):
        from paper_2512_07993_amd.build import build_library
        build_library()
    yield


def _make(struct, base, kw):
    d = dict(base, **kw)
    return struct(*[d[f[0]] for f in struct._fields_])


def _quant(**kw):
    return _make(B.CQuantCache, dict(k=0x1000, v=0x2000, k_exp=0x3001, v_exp=0x3101, stride_layer=100 * 16 * 8 * 128, stride_head=128,
                                     stride_block=16 * 8 * 128, stride_tok=8 * 128, n_layers=2, n_kv_heads=8, head_dim=128, batch=3,
                                     block_size=16, n_blocks=100, table_stride=40, block_table=0x4000), kw)


def _rows(**kw):
    return _make(B.CCache, dict(k=0x5000, v=0x6000, stride_layer=8 * 900 * 128, stride_head=900 * 128, stride_tok=128, dtype=B.BF16, n_layers=1,
                                n_kv_heads=8, n_q_heads=32, head_dim=128, batch=3, total_tokens=900, total_sentences=0, seq_off=0x7000,
                                sent_ptr=None, sent_off=None), kw)


def _queries(**kw):
    return _make(B.CQueries, dict(q=0x8000, out=0x9000, lse=None, q_stride_tok=32 * 128, q_stride_head=128, out_stride_tok=32 * 128,
                                  out_stride_head=128, dtype=B.BF16, n_q_heads=32, total_q=3, max_q=1, max_len=640, scale=0.088, q_off=0xA000), kw)


def _pages(**kw):
    return _make(B.CPages, dict(block_table=0x1000, n_held=0x2000, free_list=0x3000, n_free=0x4000, batch=3, table_stride=40, block_size=16,
                                n_blocks=100), kw)


BAD_QUANT = [
    (dict(head_dim=64), B.ECAPACITY), (dict(block_size=24), B.ECAPACITY), (dict(block_size=256), B.ECAPACITY), (dict(block_size=0), B.ECAPACITY),
    (dict(k=None), B.EINVAL), (dict(v=0x2008), B.EINVAL), (dict(k_exp=None), B.EINVAL), (dict(block_table=None), B.EINVAL),
    (dict(n_blocks=0), B.EINVAL), (dict(stride_tok=64), B.EINVAL), (dict(stride_tok=136), B.EINVAL), (dict(stride_head=8), B.EINVAL),
    (dict(stride_block=16 * 8 * 128 - 16), B.EINVAL), (dict(stride_layer=-16), B.EINVAL), (dict(batch=-1), B.EINVAL),
    (dict(batch=65536), B.ECAPACITY), (dict(table_stride=1 << 27), B.ECAPACITY), (dict(stride_tok=1 << 25, stride_block=1 << 40), B.ECAPACITY),
    (dict(n_layers=5000), B.ECAPACITY),
]


@pytest.mark.parametrize("kw,expect", BAD_QUANT)
def test_bad_cache_descriptions(kw, expect):
    lib, qc = B.lib(), _quant(**kw)
    out = C.c_size_t(0)
    batch = kw.get("batch", 3)
    for call in (lib.skipkv_quant_store, lib.skipkv_quant_load):
        assert call(C.byref(qc), C.byref(_rows(batch=batch)), 0, None, None, None, None) == expect
    assert lib.skipkv_quant_attend_workspace_bytes(C.byref(qc), C.byref(_queries()), C.byref(out)) == expect
    assert lib.skipkv_quant_attend(C.byref(qc), 0, C.byref(_queries()), 0xB000, None, None, 0, None) == expect


@pytest.mark.parametrize("kw,layer,expect", [
    (dict(n_kv_heads=4), 0, B.EINVAL), (dict(batch=2), 0, B.EINVAL), (dict(n_layers=2), 1, B.EINVAL), ({}, 2, B.EINVAL), ({}, -1, B.EINVAL),
    (dict(dtype=3), 0, B.EINVAL), (dict(k=0x5004), 0, B.EINVAL), (dict(stride_tok=132), 0, B.EINVAL), (dict(head_dim=64), 0, B.ECAPACITY),
    (dict(seq_off=None), 0, B.EINVAL),
])
def test_bad_rows(kw, layer, expect):
    lib, qc = B.lib(), _quant()
    for call in (lib.skipkv_quant_store, lib.skipkv_quant_load):
        assert call(C.byref(qc), C.byref(_rows(**kw)), layer, None, None, None, None) == expect
        assert call(None, C.byref(_rows()), 0, None, None, None, None) == B.EINVAL
        assert call(C.byref(qc), None, 0, None, None, None, None) == B.EINVAL


@pytest.mark.parametrize("kw,expect", [
    (dict(dtype=2), B.EINVAL), (dict(total_q=-1), B.EINVAL), (dict(max_q=-1), B.EINVAL), (dict(max_len=-1), B.EINVAL),
    (dict(n_q_heads=30), B.EINVAL), (dict(n_q_heads=0), B.EINVAL), (dict(n_q_heads=72), B.ECAPACITY), (dict(q_stride_tok=4), B.EINVAL),
    (dict(q_stride_head=-8), B.EINVAL), (dict(out_stride_head=64), B.EINVAL), (dict(out_stride_tok=12), B.EINVAL),
    (dict(scale=float("inf")), B.EINVAL), (dict(scale=float("nan")), B.EINVAL),
])
def test_bad_queries(kw, expect):
    lib, qc = B.lib(), _quant()
    out = C.c_size_t(0)
    assert lib.skipkv_quant_attend_workspace_bytes(C.byref(qc), C.byref(_queries(**kw)), C.byref(out)) == expect
    assert lib.skipkv_quant_attend(C.byref(qc), 0, C.byref(_queries(**kw)), 0xB000, None, None, 0, None) == expect


def test_attention_refuses_bad_pointers_layers_and_workspaces():
    lib, qc = B.lib(), _quant(table_stride=4000)
    big = _queries(max_len=64000)
    out = C.c_size_t(0)
    assert lib.skipkv_quant_attend_workspace_bytes(C.byref(qc), C.byref(big), C.byref(out)) == B.OK and out.value > 0
    need = out.value
    go = lambda q=big, layer=0, ln=0xB000, ws=0x10000, n=need: lib.skipkv_quant_attend(C.byref(qc), layer, C.byref(q), ln, None, ws, n, None)
    assert go(ln=None) == B.EINVAL and go(layer=2) == B.EINVAL and go(layer=-1) == B.EINVAL
    assert go(ws=None) == B.EWORKSPACE and go(ws=0x10010) == B.EWORKSPACE and go(n=need - 1) == B.EWORKSPACE
    for kw in (dict(q=None), dict(q=0x8008), dict(out=None), dict(out=0x9002), dict(out=0x8000), dict(q_off=None)):
        assert go(q=_queries(max_len=64000, **kw)) == B.EINVAL
    assert lib.skipkv_quant_attend(C.byref(qc), 0, None, 0xB000, None, None, 0, None) == B.EINVAL
    # a bound above what a table row holds is no larger problem than that
    assert lib.skipkv_quant_attend_workspace_bytes(C.byref(qc), C.byref(_queries(max_len=2 ** 31 - 1)), C.byref(out)) == B.OK and out.value == need
    # more workgroups than a launch can have
    wide = _queries(total_q=2 ** 31 - 1, max_q=2 ** 28, max_len=64000)
    assert lib.skipkv_quant_attend_workspace_bytes(C.byref(qc), C.byref(wide), C.byref(out)) == B.ECAPACITY


@pytest.mark.parametrize("kw,expect", [
    (dict(batch=-1), B.EINVAL), (dict(batch=4097), B.ECAPACITY), (dict(block_size=0), B.EINVAL), (dict(n_blocks=0), B.EINVAL),
    (dict(table_stride=-1), B.EINVAL), (dict(block_table=None), B.EINVAL), (dict(n_held=None), B.EINVAL), (dict(free_list=None), B.EINVAL),
    (dict(n_free=None), B.EINVAL), (dict(n_blocks=1 << 28, block_size=16), B.ECAPACITY),
])
def test_bad_pages(kw, expect):
    lib, pg = B.lib(), _pages(**kw)
    out = C.c_size_t(0)
    assert lib.skipkv_pages_workspace_bytes(C.byref(pg), C.byref(out)) == expect
    assert lib.skipkv_pages_update(C.byref(pg), 0x5000, 1, 0x6000, 3, 0x7000, None, 0x10000, 1 << 20, None) == expect


def test_pages_update_refuses_bad_arguments():
    lib, pg = B.lib(), _pages()
    out = C.c_size_t(0)
    assert lib.skipkv_pages_workspace_bytes(C.byref(pg), C.byref(out)) == B.OK and out.value > 0
    go = lambda ln=0x5000, rows=1, off=0x6000, new=3, ws=0x10000, n=out.value: lib.skipkv_pages_update(
        C.byref(pg), ln, rows, off, new, 0x7000, None, ws, n, None)
    assert go(ln=None) == B.EINVAL and go(rows=0) == B.EINVAL and go(new=-1) == B.EINVAL and go(off=None) == B.EINVAL
    assert go(ws=None) == B.EWORKSPACE and go(ws=0x10010) == B.EWORKSPACE and go(n=out.value - 1) == B.EWORKSPACE
    assert lib.skipkv_pages_update(None, 0x5000, 1, None, 0, None, None, 0x10000, 1 << 20, None) == B.EINVAL


def test_empty_calls_are_accepted_without_launching():
    lib = B.lib()
    assert lib.skipkv_pages_update(C.byref(_pages(batch=0)), None, 1, None, 0, None, None, None, 0, None) == B.OK
    assert lib.skipkv_quant_store(C.byref(_quant()), C.byref(_rows(total_tokens=0, k=None, v=None)), 0, None, None, None, None) == B.OK
    assert lib.skipkv_quant_load(C.byref(_quant(batch=0)), C.byref(_rows(batch=0)), 0, None, None, None, None) == B.OK
    assert lib.skipkv_quant_attend(C.byref(_quant()), 0, C.byref(_queries(total_q=0, q=None, out=None)), None, None, None, 0, None) == B.OK


# ---- the plain forms themselves ---------------------------------------------------------------------------------

def test_plain_encoding_rounds_to_the_nearest_code_ties_to_even():
    fine = np.array([c for c in range(256) if c not in (0x7F, 0xFF)])
    np.testing.assert_array_equal(encode(VALUES[fine], 127), fine)           # every value is its own code (and -0 keeps its sign)
    mid = (VALUES[:126] + VALUES[1:127]) / 2
    assert (encode(mid, 127) % 2 == 0).all()
    np.testing.assert_array_equal(encode(np.nextafter(mid, 1e9), 127), np.arange(1, 127))
    np.testing.assert_array_equal(encode(np.nextafter(mid, -1e9), 127), np.arange(0, 126))
    assert encode(np.array([np.nan, np.inf, -np.inf]), 127).tolist() == [0x7F] * 3


def test_plain_scale_is_the_least_power_of_two_that_holds_the_block():
    for x, byte in ((448.0, 127), (448.1, 128), (224.0, 126), (1.75, 119), (1.7500001, 120), (1.0, 119), (0.0, 1), (1e-45, 1), (3.4e38, 247)):
        assert scale_byte(np.array([x, np.inf, np.nan])) == byte, x


def test_plain_store_keeps_or_raises_the_scale_of_a_block_in_use():
    p = Pool(1, 2, 16, 1)
    p.store(0, 0, [1, 0], 16, 0, np.full((3, 128), 1.0))
    p.store(0, 0, [1, 0], 16, 3, np.full((1, 128), 0.5))
    assert p.byte[0, 0, 1] == 119
    p.store(0, 0, [1, 0], 16, 4, np.full((14, 128), 1000.0))
    assert p.byte[0, 0, 1] == 129 and p.byte[0, 0, 0] == 129
    rows = p.rows(0, 0, [1, 0], 16, 18)
    assert (rows[:3] == 1).all() and (rows[3] == 0.5).all() and (np.abs(rows[4:] - 1000) <= 1000 * 2.0 ** -4).all()
