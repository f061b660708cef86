"""Storing rows into the 8-bit cache and loading them back, against the plain 64-bit form: codes and scale bytes are the
same bits, loaded values are the values that they stand for, rounded once."""
import numpy as np
import pytest
import torch

from paper_2512_07993_amd import binding as B

from quant_helpers import D, VALUES, Pool, on_device, random_table

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _rows_of(rng, shape, dtype):
    """Rows as a cache holds them: ordinary values, some channels far larger, whole rows tiny, zero or huge."""
    x = rng.standard_normal(shape)
    x[..., ::37] *= 30
    x *= np.exp2(rng.integers(-40, 30, shape[:-1] + (1,)) * (rng.random(shape[:-1] + (1,)) < 0.1))
    x[rng.random(shape[:-1]) < 0.03] = 0.0
    return torch.from_numpy(x).to(dtype)


def _case(rng, layers, heads, lens, counts, bs, dtype, first=0, layers_all=None, width=None):
    """Pools with `lens` [layers, heads, batch] positions in use, and packed new rows of `counts` per sequence."""
    batch = len(counts)
    layers_all = layers_all or layers
    need = [-(-(int(lens[:, :, b].max()) + counts[b]) // bs) for b in range(batch)]
    table, blocks, _ = random_table(rng, need, width=width)
    pools = []
    for _ in range(2):
        p = Pool(layers_all, blocks, bs, heads)
        p.codes[:] = rng.integers(0, 256, p.codes.shape)       # slots that nobody wrote hold anything, NaN codes among it
        p.byte[:] = rng.integers(110, 140, p.byte.shape)
        pools.append(p)
    total = int(np.sum(counts))
    new = [_rows_of(rng, (layers, heads, total, D), dtype) for _ in range(2)]
    off = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    return table, pools, new, off


def _cuda(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def _store_plain(pools, new, table, bs, lens, counts, off, first):
    for p, x in zip(pools, new):
        x64 = x.double().numpy()
        for l in range(x64.shape[0]):
            for h in range(x64.shape[1]):
                for b, n in enumerate(counts):
                    if n:
                        p.store(first + l, h, table[b], bs, int(lens[l, h, b]), x64[l, h, off[b]:off[b] + n])


def _same_codes(got, ref, what):
    nan = (got & 0x7F) == 0x7F
    np.testing.assert_array_equal(nan, (ref & 0x7F) == 0x7F, err_msg=what + ": NaN")
    np.testing.assert_array_equal(got[~nan], ref[~nan], err_msg=what)


@pytest.mark.parametrize("bs", [16, 32, 64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["slots", "heads"])
def test_store_appends_at_every_place_of_a_block(bs, dtype, layout):
    rng = np.random.default_rng(bs)
    counts = [1, 0, 5, bs, bs + 1, 3 * bs + 7, 1, 2]
    lens = rng.integers(0, 2 * bs + 3, (2, 3, len(counts)))
    lens[0, 0] = [0, 0, bs - 5, bs, 1, 0, bs - 1, 2 * bs - 1]
    table, pools, new, off = _case(rng, 2, 3, lens, counts, bs, DT[dtype], layers_all=4)
    qc = on_device(*pools, table, heads_before_slots=layout == "heads", pad_blocks=2 if layout == "slots" else 0)
    k, v = (x.cuda() for x in new)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    rows = B.Cache(k, v, 3, _cuda(off), None, None, int(off[-1]), 0)
    before = [(p.codes.copy(), p.byte.copy()) for p in pools]
    B.skipkv_quant_store(qc, rows, 1, _cuda(lens.astype(np.int32)), None, status)
    torch.cuda.synchronize()
    _store_plain(pools, new, table, bs, lens, counts, off, 1)
    for name, codes, byte, p, was in (("K", qc.k, qc.k_exp, pools[0], before[0]), ("V", qc.v, qc.v_exp, pools[1], before[1])):
        np.testing.assert_array_equal(byte.cpu().numpy(), p.byte, err_msg=name)
        _same_codes(codes.cpu().numpy(), p.codes, name)
        np.testing.assert_array_equal(codes.cpu().numpy()[[0, 3]], was[0][[0, 3]])    # other layers: not a byte
    assert int(status.item()) == 0
    # storing the same rows at the same place again changes nothing
    codes, byte = qc.k.clone(), qc.k_exp.clone()
    B.skipkv_quant_store(qc, rows, 1, _cuda(lens.astype(np.int32)), None, status)
    assert torch.equal(codes, qc.k) and torch.equal(byte, qc.k_exp)


@pytest.mark.parametrize("bs", [16, 128])
def test_store_of_whole_heads_leaves_what_lies_behind_them(bs):
    # begin = NULL, end = the heads' own lengths: a compacted cache.  Strided rows, one head without a token.
    rng = np.random.default_rng(7)
    room = [70, 1, 200, 33]
    off = np.concatenate([[0], np.cumsum(room)]).astype(np.int32)
    lens = np.stack([np.stack([rng.integers(0, r + 1, 2) for r in room], axis=1)])           # [1, 2, 4]
    lens[0, 0, 2] = 0
    lens[0, 1] = room
    table, blocks, _ = random_table(rng, [-(-r // bs) for r in room])
    pools = [Pool(1, blocks, bs, 2, fill=0x7F) for _ in range(2)]
    wide = torch.randn((1, 2, sum(room), 3 * D), generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    k, v = wide[..., :D], wide[..., 2 * D:]
    qc = on_device(*pools, table, dtype=torch.float8_e4m3fn)
    B.skipkv_quant_store(qc, B.Cache(k, v, 2, _cuda(off), None, None, sum(room), 0), 0, None, _cuda(lens.astype(np.int32)))
    for p, x in zip(pools, (k, v)):
        for h in range(2):
            for b in range(4):
                p.store(0, h, table[b], bs, 0, x[0, h, off[b]:off[b] + lens[0, h, b]].double().cpu().numpy())
    for codes, byte, p in ((qc.k, qc.k_exp, pools[0]), (qc.v, qc.v_exp, pools[1])):
        np.testing.assert_array_equal(codes.view(torch.uint8).cpu().numpy(), p.codes)
        np.testing.assert_array_equal(byte.cpu().numpy(), p.byte)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_infinities_and_nan_are_stored_as_nan_and_do_not_scale_their_block(dtype):
    rng = np.random.default_rng(3)
    lens = np.zeros((1, 1, 1), dtype=np.int64)
    table, pools, new, off = _case(rng, 1, 1, lens, [48], 16, DT[dtype])
    new[0][0, 0, 3, 5], new[0][0, 0, 20, 7], new[0][0, 0, 21] = float("inf"), float("nan"), -float("inf")
    new[1][0, 0, 32:48] = float("nan")
    new[1][0, 0, 0:16] = 0.0
    qc = on_device(*pools, table)
    B.skipkv_quant_store(qc, B.Cache(new[0].cuda(), new[1].cuda(), 1, _cuda(off), None, None, 48, 0), 0, None, None)
    _store_plain(pools, new, table, 16, lens, [48], off, 0)
    for codes, byte, p in ((qc.k, qc.k_exp, pools[0]), (qc.v, qc.v_exp, pools[1])):
        np.testing.assert_array_equal(byte.cpu().numpy(), p.byte)
        _same_codes(codes.cpu().numpy(), p.codes, dtype)


def test_values_at_the_ends_of_the_types():
    # the largest fp32, the smallest normal and subnormal ones, ties between codes, and a block that falls among its subnormals
    x = torch.zeros((1, 1, 64, D), dtype=torch.float32)
    x[0, 0, 0, 0] = torch.finfo(torch.float32).max
    x[0, 0, 16, :64] = 2.0 ** -126
    x[0, 0, 17, :64] = 2.0 ** -149
    mids = torch.from_numpy((VALUES[:126] + VALUES[1:127]) / 2).float()
    x[0, 0, 32, 0], x[0, 0, 33, :126], x[0, 0, 34, :126] = 448.0, mids, -mids
    x[0, 0, 48, 0] = 448.0
    x[0, 0, 49, :D] = torch.logspace(-14, -1, D, base=2.0)
    table = np.array([[2, 0, 3, 1]], dtype=np.int32)
    pools = [Pool(1, 4, 16, 1) for _ in range(2)]
    qc = on_device(*pools, table)
    off = _cuda(np.array([0, 64], dtype=np.int32))
    B.skipkv_quant_store(qc, B.Cache(x.cuda(), x.cuda(), 1, off, None, None, 64, 0), 0, None, None)
    for p in pools:
        p.store(0, 0, table[0], 16, 0, x[0, 0].double().numpy())
    np.testing.assert_array_equal(qc.k.cpu().numpy(), pools[0].codes)
    np.testing.assert_array_equal(qc.v_exp.cpu().numpy(), pools[1].byte)
    back = torch.empty_like(x).cuda()
    B.skipkv_quant_load(qc, B.Cache(back, back.clone(), 1, off, None, None, 64, 0), 0, None, None)
    with np.errstate(under="ignore"):
        np.testing.assert_array_equal(back[0, 0].cpu().numpy(), pools[0].rows(0, 0, table[0], 16, 64).astype(np.float32))


@pytest.mark.parametrize("bs,dtype", [(16, "bf16"), (32, "f32"), (64, "bf16"), (128, "f32")])
def test_load_gives_the_values_and_writes_no_other_row(bs, dtype):
    rng = np.random.default_rng(bs + 1)
    room = [3 * bs + 5, 1, 0, 40]
    lens = np.stack([np.stack([rng.integers(0, r + 1, 3) for r in room], axis=1) for _ in range(2)])
    lens[0, 0] = room
    begin = np.minimum(rng.integers(0, bs, lens.shape), lens)
    table, blocks, _ = random_table(rng, [max(1, -(-r // bs)) for r in room])
    pools = []
    for _ in range(2):
        p = Pool(2, blocks, bs, 3)
        p.codes[:] = rng.integers(0, 256, p.codes.shape)
        p.byte[:] = rng.integers(100, 150, p.byte.shape)
        pools.append(p)
    qc = on_device(*pools, table, heads_before_slots=bs == 32)
    off = np.concatenate([[0], np.cumsum(room)]).astype(np.int32)
    for first in (None, begin):
        k = torch.full((2, 3, sum(room), D), -7.0, dtype=DT[dtype], device="cuda")
        v = k.clone()
        B.skipkv_quant_load(qc, B.Cache(k, v, 3, _cuda(off), None, None, sum(room), 0), 0,
                            None if first is None else _cuda(first.astype(np.int32)), _cuda(lens.astype(np.int32)))
        for got, p in ((k, pools[0]), (v, pools[1])):
            want = torch.full_like(got, -7.0).cpu()
            for l in range(2):
                for h in range(3):
                    for b in range(4):
                        lo = 0 if first is None else int(first[l, h, b])
                        n = int(lens[l, h, b])
                        want[l, h, off[b]:off[b] + n - lo] = torch.from_numpy(p.rows(l, h, table[b], bs, n)[lo:]).to(DT[dtype])
            assert torch.equal(torch.nan_to_num(got.float(), nan=12345.0), torch.nan_to_num(want.float(), nan=12345.0).cuda())


def test_values_keep_their_bits_through_load_and_store_into_other_blocks():
    # what a compression step does to the cache: rows of one block come to lie among those of another
    rng = np.random.default_rng(11)
    x = torch.from_numpy(rng.standard_normal((1, 4, 500, D))).bfloat16()
    table, blocks, _ = random_table(rng, [32])
    qc = on_device(Pool(1, blocks, 16, 4), Pool(1, blocks, 16, 4), table)
    off = _cuda(np.array([0, 500], dtype=np.int32))
    a, a2 = x.cuda(), (x * 3).cuda()
    cache = B.Cache(a, a2, 4, off, None, None, 500, 0)
    B.skipkv_quant_store(qc, cache, 0, None, None)
    B.skipkv_quant_load(qc, cache, 0, None, None)
    kept = torch.from_numpy(np.sort(rng.choice(500, 203, replace=False))).cuda()
    b = torch.zeros_like(a)
    b[:, :, :203] = a[:, :, kept]
    b2 = torch.zeros_like(a2)
    b2[:, :, :203] = a2[:, :, kept]
    ln = torch.full((1, 4, 1), 203, dtype=torch.int32, device="cuda")
    again = B.Cache(b.clone(), b2.clone(), 4, off, None, None, 500, 0)
    B.skipkv_quant_store(qc, again, 0, None, ln)
    B.skipkv_quant_load(qc, again, 0, None, ln)
    # N(0,1) rows: every block's scale is within a factor of 4 of another's, so values from 2^-6 of the largest scale up are exact
    for got, want in ((again.k, b), (again.v, b2)):
        big = want.abs() >= 2.0 ** -6 * 2.0 ** (int(torch.stack([qc.k_exp.max(), qc.v_exp.max()]).max()) - 127)
        assert torch.equal(got[big], want[big])
        assert float((got - want)[~big].float().abs().max()) <= 2.0 ** -10 * 2.0 ** (int(torch.stack([qc.k_exp.max(), qc.v_exp.max()]).max()) - 127)


def test_ranges_and_blocks_that_do_not_fit_are_skipped_and_reported():
    rng = np.random.default_rng(5)
    counts = [20, 20, 20, 20]
    lens = np.zeros((1, 2, 4), dtype=np.int64)
    table, pools, new, off = _case(rng, 1, 2, lens, counts, 16, torch.bfloat16, width=4)
    table[2, 1] = 10 ** 6                                # sequence 2: its second block is no block
    qc = on_device(*pools, table)
    rows = B.Cache(new[0].cuda(), new[1].cuda(), 2, _cuda(off), None, None, 80, 0)
    begin = np.zeros((1, 2, 4), dtype=np.int32)
    end = np.full((1, 2, 4), 20, dtype=np.int32)
    begin[0, 0, 0] = -1                                  # head 0: before the start, backwards, and longer than the rows
    begin[0, 1, 1], end[0, 1, 1] = 21, 20
    end[0, 1, 3] = 21
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.skipkv_quant_store(qc, rows, 0, _cuda(begin), _cuda(end), status)
    assert int(status.item()) == B.DEV_BAD_LENGTHS | B.DEV_BAD_BLOCK_TABLE
    for p, x in zip(pools, new):
        for h in range(2):
            for b in range(4):
                if (h, b) in ((0, 0), (1, 1), (1, 3)):
                    continue
                n = 16 if b == 2 else 20
                p.store(0, h, table[b], 16, 0, x[0, h, off[b]:off[b] + n].double().numpy())
    np.testing.assert_array_equal(qc.k.cpu().numpy(), pools[0].codes)
    np.testing.assert_array_equal(qc.v_exp.cpu().numpy(), pools[1].byte)
    # the load, and an end beyond the table row
    status.zero_()
    k = torch.full((1, 2, 80, D), -7.0, dtype=torch.bfloat16, device="cuda")
    cache = B.Cache(k, k.clone(), 2, _cuda(off), None, None, 80, 0)
    B.skipkv_quant_load(qc, cache, 0, _cuda(begin), _cuda(end), status)
    assert int(status.item()) == B.DEV_BAD_LENGTHS | B.DEV_BAD_BLOCK_TABLE
    assert bool((k[0, 0, 0:20] == -7).all()) and bool((k[0, 1, 20:40] == -7).all()) and bool((k[0, 1, 60:80] == -7).all())
    assert bool((k[0, :, 56:60] == -7).all()) and not bool((k[0, :, 40:56] == -7).any())
    status.zero_()
    far = torch.full((1, 2, 4), 60, dtype=torch.int32, device="cuda")   # 60 + 20 > 4 * 16
    B.skipkv_quant_store(qc, rows, 0, far, None, status)
    assert int(status.item()) == B.DEV_BAD_LENGTHS
    np.testing.assert_array_equal(qc.k.cpu().numpy(), pools[0].codes)
