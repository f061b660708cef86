"""Attention over the 8-bit cache against a plain form in 64 bits, at the sizes, masks, layouts and contents where it can go
wrong.  The bounds are derived in quant_helpers.attend_reference."""
import math

import numpy as np
import pytest
import torch

from paper_2512_07993_amd import binding as B

from quant_helpers import D, U_OUT, Pool, attend_reference, check_close, encode, on_device, random_table, scale_byte

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
SCALE = 1 / math.sqrt(D)
# what the weights are rounded to for the second product: bf16 outputs one bf16 number with more than 16 query rows per
# KV head, else two (2^-16); fp32 outputs three (2^-24)
ONE_PART, TWO_PARTS, THREE_PARTS = 2.0 ** -8, 2.0 ** -16, 2.0 ** -24


def parts_of(dtype, max_q, group):
    return THREE_PARTS if dtype == "f32" else TWO_PARTS if max_q * group <= 16 else ONE_PART


def _cuda(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def fill(rng, pool, l, h, table, bs, n, size=1.0):
    x = rng.standard_normal((n, D)) * size
    x[:, ::29] *= 4
    pool.store(l, h, table, bs, 0, x)


def build(rng, heads, lens, bs, layers=1, width=None, behind=0x7F):
    """Pools holding `lens` [layers, heads, batch] tokens; slots behind them hold NaN codes."""
    batch = lens.shape[2]
    counts = [-(-int(lens[:, :, b].max()) // bs) for b in range(batch)]
    table, blocks, _ = random_table(rng, counts, width=width or max(1, max(counts)) + 1)
    k, v = (Pool(layers, blocks, bs, heads, fill=behind) for _ in range(2))
    for l in range(layers):
        for h in range(heads):
            for b in range(batch):
                if lens[l, h, b]:
                    fill(rng, k, l, h, table[b], bs, int(lens[l, h, b]), 0.5 + h)
                    fill(rng, v, l, h, table[b], bs, int(lens[l, h, b]), 2.0 ** (b % 5 - 2))
    return k, v, table


def run(qc, layer, q, ms, lens, dtype, max_len=None, max_q=None, lse=True, stream=None, scale=SCALE):
    off = np.concatenate([[0], np.cumsum(ms)]).astype(np.int32)
    out = torch.full((q.shape[0], q.shape[1], D), 99.0, dtype=q.dtype, device="cuda")
    ls = torch.full((q.shape[0], q.shape[1]), 99.0, device="cuda") if lse else None
    qs = B.Queries(q, out, _cuda(off), max_q=max(ms) if max_q is None else max_q, max_len=int(lens.max()) if max_len is None else max_len,
                   scale=scale, lse=ls)
    ws = torch.empty(B.skipkv_quant_attend_workspace_bytes(qc, qs) + 256, dtype=torch.uint8, device="cuda").fill_(0xFF)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.skipkv_quant_attend(qc, layer, qs, _cuda(lens.astype(np.int32)), ws, status, stream)
    torch.cuda.synchronize()
    return out, ls, int(status.item())


def check(out, lse, q, ms, lens, k, v, table, bs, layer, parts, heads=None, scale=SCALE):
    hk, g = lens.shape[0], q.shape[1] // lens.shape[0]
    qn = q.double().cpu().numpy()
    got, gl = out.double().cpu().numpy(), None if lse is None else lse.double().cpu().numpy()
    at = 0
    for b, m in enumerate(ms):
        for h in range(hk) if heads is None else heads:
            n = int(lens[h, b])
            if m == 0:
                continue
            ref, rl, tol, ltol = attend_reference(qn[at:at + m, h * g:(h + 1) * g], k.rows(layer, h, table[b], bs, n),
                                                  v.rows(layer, h, table[b], bs, n), m, scale, parts)
            what = "sequence %d head %d: %d keys, %d queries" % (b, h, n, m)
            check_close(got[at:at + m, h * g:(h + 1) * g], ref, tol + U_OUT[out.dtype] * (np.abs(ref) + tol), what)
            if gl is not None:
                check_close(gl[at:at + m, h * g:(h + 1) * g], rl, ltol, "lse, " + what)
        at += m


def queries(rng, total, heads, dtype):
    return torch.from_numpy(rng.standard_normal((total, heads, D)) * 1.5).to(DT[dtype]).cuda()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("group", [1, 2, 3, 4, 5, 7, 8])
def test_single_tokens_at_lengths_around_tiles_and_blocks(dtype, group):
    rng = np.random.default_rng(group)
    bs = [16, 32, 64, 128][group % 4]
    lens = np.array([[0, 1, 15, 16, 17, 31, 32, 33, 64, 127, 128, 129, 255, 256, 257, 300]]).repeat(2, 0)
    lens[1] = lens[1][::-1]
    k, v, table = build(rng, 2, lens[None], bs)
    q = queries(rng, 16, 2 * group, dtype)
    out, lse, status = run(on_device(k, v, table), 0, q, [1] * 16, lens, dtype)
    assert status == 0
    check(out, lse, q, [1] * 16, lens, k, v, table, bs, 0, parts_of(dtype, 1, group))
    assert bool((out[0, :group] == 0).all()) and bool(torch.isneginf(lse[0, :group]).all())     # nothing to see


@pytest.mark.parametrize("dtype,group,bs,ms", [
    ("bf16", 4, 16, [1, 4, 2, 0, 3]), ("bf16", 4, 32, [5, 0, 17, 33, 1]), ("bf16", 8, 16, [70, 1, 64, 5, 129]), ("bf16", 1, 64, [16, 31, 64, 1, 200]),
    ("bf16", 7, 128, [9, 40, 3, 100, 77]), ("bf16", 5, 16, [2, 3, 1, 2, 3]), ("f32", 4, 16, [4, 1, 9, 0, 30]), ("f32", 7, 64, [2, 19, 5, 1, 8])])
def test_several_tokens_see_up_to_their_own_position(dtype, group, bs, ms):
    rng = np.random.default_rng(sum(ms))
    lens = np.array([[ms[0], 150, 33, 7, 290], [40, ms[1] + 1, 500, 64, 130]])
    lens = np.maximum(lens, np.array(ms)[None, :] - 2)            # in places two queries stand before the first key
    k, v, table = build(rng, 2, lens[None], bs)
    q = queries(rng, sum(ms), 2 * group, dtype)
    out, lse, status = run(on_device(k, v, table), 0, q, ms, lens, dtype)
    assert status == 0
    check(out, lse, q, ms, lens, k, v, table, bs, 0, parts_of(dtype, max(ms), group))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m", [1, 3, 40])
def test_long_caches_are_cut_and_joined(dtype, m):
    rng = np.random.default_rng(m)
    lens = np.array([[9001, 300, 4097], [1, 5000, 8192]])
    lens = np.maximum(lens, m)
    k, v, table = build(rng, 2, lens[None], 16)
    ms = [m, 1, m]
    q = queries(rng, sum(ms), 8, dtype)
    qc = on_device(k, v, table)
    out, lse, status = run(qc, 0, q, ms, lens, dtype)
    assert status == 0
    check(out, lse, q, ms, lens, k, v, table, 16, 0, parts_of(dtype, m, 4))
    again, lse2, _ = run(qc, 0, q, ms, lens, dtype)
    assert torch.equal(out, again) and torch.equal(lse, lse2)     # the same bits every time


def test_bounds_above_the_lengths_only_change_the_order_of_additions():
    rng = np.random.default_rng(17)
    lens = np.array([[700, 20, 31]])
    k, v, table = build(rng, 1, lens[None], 32, width=400)
    q = queries(rng, 3, 4, "bf16")
    qc = on_device(k, v, table)
    for max_len, max_q in ((700, 1), (12800, 1), (2 ** 31 - 1, 1), (5000, 4)):
        out, lse, status = run(qc, 0, q, [1, 1, 1], lens, "bf16", max_len=max_len, max_q=max_q)
        assert status == 0
        check(out, lse, q, [1, 1, 1], lens, k, v, table, 32, 0, parts_of("bf16", min(max_q, 3), 4))


@pytest.mark.parametrize("layout", ["heads", "padded", "e4m3"])
def test_layouts_strides_and_layers(layout):
    rng = np.random.default_rng(23)
    lens = rng.integers(1, 200, (3, 4, 5))
    k, v, table = build(rng, 4, lens, 16, layers=3)
    qc = on_device(k, v, table, heads_before_slots=layout == "heads", pad_blocks=3 if layout == "padded" else 0,
                   dtype=torch.float8_e4m3fn if layout == "e4m3" else torch.uint8)
    ms = [2, 1, 3, 1, 2]
    # q lies among keys and values of one projection, tokens with gaps; out has its heads first
    wide = queries(rng, sum(ms), 16 + 8, "bf16")
    q = wide[:, 4:20]
    off = np.concatenate([[0], np.cumsum(ms)]).astype(np.int32)
    for layer in (0, 2):
        out = torch.full((16, sum(ms), D), 99.0, dtype=torch.bfloat16, device="cuda").transpose(0, 1)
        qs = B.Queries(q, out, _cuda(off), max_q=3, max_len=200, scale=0.11)
        ws = torch.empty(B.skipkv_quant_attend_workspace_bytes(qc, qs) + 256, dtype=torch.uint8, device="cuda")
        B.skipkv_quant_attend(qc, layer, qs, _cuda(lens[layer].astype(np.int32)), ws)
        check(out, None, q, ms, lens[layer], k, v, table, 16, layer, parts_of("bf16", 3, 4), scale=0.11)


@pytest.mark.parametrize("m,group", [(6, 2), (24, 2), (64, 4), (12, 2)])
def test_nan_values_reach_exactly_the_queries_that_see_them(m, group):
    rng = np.random.default_rng(29)
    bs = 16
    lens = np.array([[200, 77]])
    k, v, table = build(rng, 1, lens[None], bs)
    def poke(pool, b, t, d):
        pool.codes[0, table[b, t // bs], t % bs, 0, d] = 0xFF if d % 2 else 0x7F
    for d in (0, 5, 64, 127):
        poke(v, 0, 200 - 2, d)                   # seen by the last two queries
        poke(v, 1, 77 - 1, d)                    # by the last one
    poke(v, 1, 77 - m + 1, 3)                    # by all but the first
    poke(k, 0, 200 - 1, 9)                       # a key: the last query's whole row
    poke(v, 0, 3, 77)                            # by all
    q = queries(rng, 2 * m, group, "bf16")
    out, lse, status = run(on_device(k, v, table), 0, q, [m, m], lens, "bf16")
    assert status == 0
    check(out, lse, q, [m, m], lens, k, v, table, bs, 0, parts_of("bf16", m, group))
    bad = torch.isnan(out).any(1).cpu().numpy()  # [tokens, D]
    assert bad[:m - 2].sum() == m - 2 and bad[m - 2, [0, 5, 64, 77, 127]].all() and bad[m - 2].sum() == 5 and bad[m - 1].all()
    assert not bad[m].any() and bad[m + 1, 3] and bad[m + 1].sum() == (1 if m > 2 else 5)


def test_a_query_with_nan_or_infinity_concerns_itself_only():
    rng = np.random.default_rng(31)
    lens = np.array([[100, 50]])
    k, v, table = build(rng, 1, lens[None], 16)
    q = queries(rng, 8, 2, "bf16")
    clean, _, _ = run(on_device(k, v, table), 0, q, [4, 4], lens, "bf16")
    q[2, 0, 7], q[5, 1, 3] = float("nan"), float("inf")
    out, lse, _ = run(on_device(k, v, table), 0, q, [4, 4], lens, "bf16")
    rows = torch.ones(8, 2, dtype=torch.bool, device="cuda")
    rows[2, 0] = rows[5, 1] = False
    assert torch.equal(out[rows], clean[rows]) and bool(torch.isnan(out[~rows]).all()) and bool(torch.isnan(lse[~rows]).all())


def test_logits_of_any_size():
    # sharp softmaxes (one key takes all), references that keep rising along the cache, and scales of both signs
    rng = np.random.default_rng(37)
    lens = np.array([[600, 70]])
    k, v, table = build(rng, 1, lens[None], 16)
    rows = k.rows(0, 0, table[0], 16, 600) * np.linspace(0.01, 20, 600)[:, None]
    k.store(0, 0, table[0], 16, 0, rows)
    q = queries(rng, 2, 4, "f32")
    for scale in (SCALE, 1.0, -2.0, 1e-6, 0.0):
        out, lse, _ = run(on_device(k, v, table), 0, q, [1, 1], lens, "f32", scale=scale)
        check(out, lse, q, [1, 1], lens, k, v, table, 16, 0, THREE_PARTS, scale=scale)


def test_blocks_of_very_different_scale_and_of_zeros():
    rng = np.random.default_rng(41)
    lens = np.array([[160]])
    k, v, table = build(rng, 1, lens[None], 16)
    for i in range(10):
        size = [1.0, 1e-30, 1e30, 0.0, 1e-3][i % 5]
        v.store(0, 0, table[0], 16, 16 * i, rng.standard_normal((16, D)) * size)
        k.store(0, 0, table[0], 16, 16 * i, rng.standard_normal((16, D)) * [1.0, 0.0, 1e-30][i % 3])
    q = queries(rng, 1, 4, "f32")
    out, lse, _ = run(on_device(k, v, table), 0, q, [1], lens, "f32")
    check(out, lse, q, [1], lens, k, v, table, 16, 0, THREE_PARTS)


def test_offsets_beyond_32_bits():
    # pools of 5 GB: the blocks in use lie at both ends
    rng = np.random.default_rng(43)
    bs, heads, blocks = 64, 8, 5 * 2 ** 30 // (64 * 8 * D)
    table = np.array([[blocks - 1, 0, blocks - 2, blocks // 2]], dtype=np.int32)
    lens = np.full((heads, 1), 250)
    small = [Pool(1, 4, bs, heads) for _ in range(2)]
    local = np.array([[0, 1, 2, 3]], dtype=np.int32)
    for p in small:
        for h in range(heads):
            fill(rng, p, 0, h, local[0], bs, 250)
    codes = [torch.empty((1, blocks, bs, heads, D), dtype=torch.uint8, device="cuda") for _ in range(2)]
    exps = [torch.empty((1, heads, blocks), dtype=torch.uint8, device="cuda") for _ in range(2)]
    off = _cuda(np.array([0, 250], dtype=np.int32))
    qc = B.QuantCache(codes[0], codes[1], exps[0], exps[1], _cuda(table))
    rows = [torch.from_numpy(np.stack([p.rows(0, h, local[0], bs, 250) for h in range(heads)])[None]).float().cuda() for p in small]
    B.skipkv_quant_store(qc, B.Cache(rows[0], rows[1], heads, off, None, None, 250, 0), 0, None, None)
    back = [torch.zeros_like(x) for x in rows]
    B.skipkv_quant_load(qc, B.Cache(back[0], back[1], heads, off, None, None, 250, 0), 0, None, None)
    assert torch.equal(back[0], rows[0]) and torch.equal(back[1], rows[1])
    q = queries(rng, 1, 4 * heads, "bf16")
    out, lse, status = run(qc, 0, q, [1], lens, "bf16")
    assert status == 0
    check(out, lse, q, [1], lens, small[0], small[1], local, bs, 0, TWO_PARTS)


def test_lengths_offsets_and_blocks_that_do_not_fit_are_reported_and_concern_their_rows_only():
    rng = np.random.default_rng(47)
    lens = np.array([[50, 60, 70, 80, 90, 100]]).repeat(2, 0)
    k, v, table = build(rng, 2, lens[None], 16, width=8)
    q = queries(rng, 6, 8, "bf16")
    clean, _, _ = run(on_device(k, v, table), 0, q, [1] * 6, lens, "bf16", max_len=100)
    bad = lens.copy()
    bad[0, 0], bad[1, 2], bad[0, 3] = -1, 101, 129          # negative, above the bound, above the table row too
    t2 = table.copy()
    t2[5, 3], t2[4, 7] = -1, 10 ** 6                         # (the second one is not among the sequence's blocks)
    out, lse, status = run(on_device(k, v, t2), 0, q, [1] * 6, bad, "bf16", max_len=100)
    assert status == B.DEV_BAD_LENGTHS | B.DEV_BAD_BLOCK_TABLE
    gone = torch.zeros(6, 2, dtype=torch.bool, device="cuda")
    gone[0, 0] = gone[2, 1] = gone[3, 0] = gone[5] = True
    o, c = out.view(6, 2, 4, D), clean.view(6, 2, 4, D)
    assert bool(torch.isnan(o[gone]).all()) and torch.equal(o[~gone], c[~gone]) and bool(torch.isnan(lse.view(6, 2, 4)[gone]).all())
    # query offsets: a sequence whose entries descend, leave the array or lie too far apart has no output
    for off in ([0, 1, 0, 3, 4, 5, 6], [0, 1, 2, 3, 4, 5, 7], [-1, 1, 2, 3, 4, 5, 6], [0, 3, 3, 3, 4, 5, 6]):
        res = torch.full_like(q, 99.0)
        qs = B.Queries(q, res, _cuda(np.array(off, dtype=np.int32)), max_q=2, max_len=100, scale=SCALE)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        ws = torch.empty(B.skipkv_quant_attend_workspace_bytes(on_device(k, v, table), qs) + 256, dtype=torch.uint8, device="cuda")
        B.skipkv_quant_attend(on_device(k, v, table), 0, qs, _cuda(lens.astype(np.int32)), ws, status)
        assert int(status.item()) == B.DEV_BAD_LENGTHS
        assert torch.equal(res[4], clean[4])


def test_many_short_sequences():
    rng = np.random.default_rng(53)
    batch = 300
    lens = rng.integers(0, 40, (1, batch))
    ms = [int(x) for x in rng.integers(0, 3, batch)]
    k, v, table = build(rng, 1, lens[None], 16)
    q = queries(rng, sum(ms), 2, "bf16")
    out, lse, status = run(on_device(k, v, table), 0, q, ms, lens, "bf16")
    assert status == 0
    check(out, lse, q, ms, lens, k, v, table, 16, 0, TWO_PARTS)


def test_on_another_stream():
    rng = np.random.default_rng(59)
    lens = np.array([[900, 30]])
    k, v, table = build(rng, 1, lens[None], 16)
    q = queries(rng, 2, 4, "bf16")
    qc = on_device(k, v, table)
    want, _, _ = run(qc, 0, q, [1, 1], lens, "bf16")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got, _, _ = run(qc, 0, q, [1, 1], lens, "bf16", stream=s)
    assert torch.equal(got, want)
