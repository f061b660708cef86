"""Attention over the 8-bit cache at the edges of what its header promises: offsets that make more work than the call has
room for, and how far results may be off."""
import numpy as np
import pytest
import torch

from paper_2512_07993_amd import binding as B

from quant_helpers import D, Pool, attend_reference, check_close, on_device
from test_quant_host import _entry_points
from test_gpu_quant_attend import SCALE, TWO_PARTS, _cuda, build, check, parts_of, queries, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fill", [0x00, 0x3C, 0xFF])
def test_rows_beyond_the_call_are_left_alone(fill):
    """Descending offsets give 101 sequences of 256 tokens where the call has 512 tokens in all.  A hundred of them are the same sequence
    (table, lengths, rows); the last one may have no output, but none that comes out of the workspace."""
    rng = np.random.default_rng(1)
    heads, group, m, n_same, width = 4, 4, 256, 100, 11
    off = np.array([0, m] * n_same + [m, 2 * m], dtype=np.int32)
    batch = len(off) - 1                                     # [0, m), descending, [0, m), ..., [0, m), empty, [m, 2 m)
    lens = np.tile(rng.integers(1000, 1400, (heads, 1)), (1, batch))
    table = np.tile(rng.integers(0, 40, (1, width)).astype(np.int32), (batch, 1))
    pools = [Pool(1, 40, 128, heads) for _ in range(2)]
    for pool in pools:
        pool.codes[:] = rng.integers(0, 127, pool.codes.shape) + 128 * rng.integers(0, 2, pool.codes.shape)
        pool.byte[:] = rng.integers(112, 119, pool.byte.shape)
    q = queries(rng, 2 * m, heads * group, "bf16")
    out, lse = torch.full_like(q, 99.0), torch.full(q.shape[:2], 99.0, device="cuda")
    qs = B.Queries(q, out, _cuda(off), max_q=m, max_len=width * 128, scale=SCALE, lse=lse)
    qc, status = on_device(*pools, table), torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = torch.empty(B.skipkv_quant_attend_workspace_bytes(qc, qs) + 256, dtype=torch.uint8, device="cuda").fill_(fill)
    B.skipkv_quant_attend(qc, 0, qs, _cuda(lens.astype(np.int32)), ws, status)
    assert int(status.item()) == B.DEV_BAD_LENGTHS
    check(out[:m], lse[:m], q[:m], [m], lens[:, :1], *pools, table[:1], 128, 0, parts_of("bf16", m, group), heads=[0, 3])
    for h in range(heads):
        mine = out[m:, group * h:group * (h + 1)]
        written = (mine != 99).any(2)
        if bool(written.any()):
            assert bool(written.all())
            check(out[m:], lse[m:], q[m:], [m], lens[:, :1], *pools, table[:1], 128, 0, parts_of("bf16", m, group), heads=[h])
        else:
            assert bool((lse[m:, group * h:group * (h + 1)] == 99).all())


# ---- two parts of a weight ----------------------------------------------------------------------------------
# Values of one sign: sum_t p_t |v_t| is the output itself, so the bound of two-part weights, 2^-16 of it, is small against a step of the
# output, and the output has to be the exact one rounded, but where that lies within the bound of a border.  (The roundings of one-part
# weights, up to 2^-8 of each, move a result of a few large weights by up to a step.)

def _half_step(x):
    return 2.0 ** (np.floor(np.log2(np.maximum(x, 2.0 ** -120))) - 8)      # bf16: 8 significant bits


def check_rounded_once(out, q, ms, lens, k, v, table, bs, heads, scale=SCALE):
    hk, g = lens.shape[0], q.shape[1] // lens.shape[0]
    qn, got = q.double().cpu().numpy(), out.double().cpu().numpy()
    at = 0
    for b, m in enumerate(ms):
        for h in heads:
            n = int(lens[h, b])
            ref, _, tol, _ = attend_reference(qn[at:at + m, h * g:(h + 1) * g], k.rows(0, h, table[b], bs, n), v.rows(0, h, table[b], bs, n), m,
                                              scale, TWO_PARTS, device=q.device)
            check_close(got[at:at + m, h * g:(h + 1) * g], ref, tol + _half_step(ref + tol), "sequence %d head %d: %d keys, %d queries" % (b, h, n, m))
        at += m


def positive(rng, heads, lens, bs):
    k, v, table = build(rng, heads, lens[None], bs)
    v.codes[:] = np.where((v.codes & 0x7F) == 0x7F, v.codes, v.codes & 0x7F)
    return k, v, table


def sharp(rng, total, heads, dtype="bf16"):
    """Queries whose weights lie on a few keys."""
    return queries(rng, total, heads, dtype) * 3


@pytest.mark.parametrize("longest", [60, 700, 5000, 20000])
@pytest.mark.parametrize("m,group", [(1, 1), (1, 4), (2, 8), (16, 1), (17, 1), (5, 4), (3, 7), (8, 4), (4, 8), (32, 1)])
def test_up_to_32_rows_take_the_weights_in_two_parts(m, group, longest):
    rng = np.random.default_rng(m * 10 + group)
    lens = np.array([[longest, max(m, longest // 7)]]).repeat(2, 0)
    lens[1] = np.maximum(m, lens[1] // 2)
    k, v, table = positive(rng, 2, lens, 64)
    q = sharp(rng, 2 * m, 2 * group)
    out, _, status = run(on_device(k, v, table), 0, q, [m, m], lens, "bf16")
    assert status == 0
    check_rounded_once(out, q, [m, m], lens, k, v, table, 64, [0, 1])


@pytest.mark.parametrize("batch,m,group", [(4, 20, 4), (4, 40, 4), (2, 9, 4)])
def test_more_rows_that_are_taken_16_or_32_at_a_time_too(batch, m, group):
    """Few sequences with so few rows that blocks of 256 would leave most CUs without work."""
    rng = np.random.default_rng(m)
    lens = np.full((8, batch), 1100) - np.arange(8)[:, None]
    k, v, table = positive(rng, 8, lens, 64)
    q = sharp(rng, batch * m, 8 * group)
    out, _, status = run(on_device(k, v, table), 0, q, [m] * batch, lens, "bf16")
    assert status == 0
    check_rounded_once(out, q, [m] * batch, lens, k, v, table, 64, [0, 5])


# ---- values that no bf16 number is ---------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,m,group,longest", [("bf16", 5, 1, 98), ("bf16", 4, 4, 5010), ("f32", 5, 2, 98), ("f32", 3, 4, 5010), ("bf16", 8, 4, 98),
                                                   ("bf16", 30, 1, 5010), ("bf16", 70, 8, 98), ("bf16", 200, 4, 210), ("bf16", 150, 4, 9010)])
def test_the_largest_numbers_reach_only_the_queries_that_see_them(dtype, m, group, longest):
    """Numbers from 248 * 2^120 on are rounded to 2^128, which is an infinity in the second product: 0 times it must not reach the queries that do not
    see it, as 0 times a NaN does not.  The last two keys are in a block of their own and hold 0 but for these dimensions."""
    rng = np.random.default_rng(m + group)
    big = torch.tensor([torch.finfo(torch.bfloat16).max, 249 * 2.0 ** 120, -448.0 * 2.0 ** 119, torch.finfo(torch.bfloat16).min]).double().numpy()
    dims, bs = [0, 29, 64, 127], 16
    lens = np.array([[longest, longest - 8]])
    k, v, table = build(rng, 1, lens[None], bs)
    rows = np.zeros((2, 128))
    rows[0, dims] = big
    rows[1, dims[0]] = big[0]
    at = longest - 2
    assert at % bs == 0
    v.store(0, 0, table[0], bs, at, rows)
    assert v.byte[0, 0, table[0, at // bs]] == 247
    ms = [m, min(m, 3)]
    q = queries(rng, sum(ms), group, dtype)
    out, lse, status = run(on_device(k, v, table), 0, q, ms, lens, dtype)
    assert status == 0
    far = [d for d in dims if d != dims[2]]                    # (448 * 2^119 is a bf16 number, and in the sums below too large to compare)
    assert bool(torch.isfinite(out[:m - 2]).all()) and bool(torch.isfinite(out[m:]).all())
    assert not bool(torch.isfinite(out[m - 2:m][:, :, far]).any())
    rest = [d for d in range(128) if d not in dims]
    assert bool(torch.isfinite(out[:, :, rest]).all())
    for d in dims:                                             # what the others see: as without those two
        v.codes[0, table[0, at // bs], :2, 0, d] = 0
    same, slse, status = run(on_device(k, v, table), 0, q, ms, lens, dtype)
    assert status == 0 and torch.equal(lse, slse)
    assert torch.equal(out[:m - 2], same[:m - 2]) and torch.equal(out[m:], same[m:]) and torch.equal(out[:, :, rest], same[:, :, rest])
    check(same, slse, q, ms, lens, k, v, table, bs, 0, parts_of(dtype, m, group))


def test_workspaces_and_status_words_elsewhere_are_refused():
    """In host memory, or with gaps: before anything is launched."""
    rng = np.random.default_rng(5)
    lens = np.array([[500, 30]])
    k, v, table = build(rng, 1, lens[None], 16)
    qc, q, n = on_device(k, v, table), queries(rng, 2, 4, "bf16"), _cuda(lens.astype(np.int32))
    off = _cuda(np.array([0, 1, 2], dtype=np.int32))
    qs = B.Queries(q, torch.zeros_like(q), off, max_q=1, max_len=500, scale=SCALE)
    pages = B.Pages(qc.block_table, _cuda(np.array([2, 2], dtype=np.int32)), torch.zeros(9, dtype=torch.int32, device="cuda"),
                    torch.zeros(1, dtype=torch.int32, device="cuda"), 16)
    rows = B.Cache(*(torch.zeros((1, 1, 2, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)), 4, off, off, off, 2, 0)
    need = B.skipkv_quant_attend_workspace_bytes(qc, qs)
    good, status = torch.empty(need, dtype=torch.uint8, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    calls = [lambda ws, st: B.skipkv_quant_attend(qc, 0, qs, n, ws, st), lambda ws, st: B.skipkv_pages_update(pages, n, off, 2, None, ws, st),
             lambda ws, st: B.skipkv_quant_store(qc, rows, 0, None, None, st), lambda ws, st: B.skipkv_quant_load(qc, rows, 0, None, None, st)]
    for call in calls[:2]:
        for ws in (good.cpu(), torch.empty(4 * need, dtype=torch.uint8, device="cuda")[::4]):
            with pytest.raises(AssertionError, match="workspace"):
                call(ws, status)
    for call in calls:
        for st in (status.cpu(), status.long()):
            with pytest.raises(AssertionError, match="status"):
                call(good, st)
    B.skipkv_quant_attend(qc, 0, qs, n, good, status)
    assert int(status.item()) == 0 and bool(torch.isfinite(qs.out).all())


@pytest.mark.parametrize("name", ["attend", "pages", "store", "load"])
def test_calls_on_tensors_in_host_memory_are_refused(name):
    with pytest.raises(AssertionError, match="host memory"):
        _entry_points()[name](torch.zeros(1 << 20, dtype=torch.uint8), None)
