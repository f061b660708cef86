"""The 8-bit cache and its attention where the kernels change their way: heads taken together, keys cut into chunks and
joined, blocks of 16 and of 256 query rows; in graphs, on two streams, with blocks that sequences share; and what the binding
refuses."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2512_07993_amd import binding as B

from quant_helpers import Pool, on_device
from test_gpu_quant_attend import SCALE, _cuda, build, check, parts_of, queries, run

pytestmark = pytest.mark.gpu
D = 128


@pytest.mark.parametrize("heads", [1, 2, 3, 4, 6, 8, 12])
@pytest.mark.parametrize("dtype,m,group", [("bf16", 1, 4), ("f32", 2, 3)])
def test_heads_of_different_length_in_cut_caches(heads, dtype, m, group):
    """Heads that a workgroup takes together end in different chunks; some have nothing in the later ones, some nothing at all."""
    rng = np.random.default_rng(100 + heads)
    lens = rng.integers(0, 5000, (heads, 2))
    lens[0, 0], lens[-1, 1] = 4999, 0
    lens[heads // 2, 0] = 1
    k, v, table = build(rng, heads, lens[None], 16)
    q = queries(rng, 2 * m, heads * group, dtype)
    out, lse, status = run(on_device(k, v, table), 0, q, [m, m], lens, dtype, max_len=5000)
    assert status == 0
    check(out, lse, q, [m, m], lens, k, v, table, 16, 0, parts_of(dtype, m, group))


DEALT = {
    "one long, others short": lambda rng, hk, n: np.where(np.arange(n)[None, :] == n // 2, 20000, rng.integers(1, 60, (hk, n))),
    "spread": lambda rng, hk, n: rng.integers(1, 20001, (hk, n)),
    "nothing anywhere": lambda rng, hk, n: np.zeros((hk, n), dtype=np.int64),
    "all the same": lambda rng, hk, n: np.full((hk, n), 6000),
    "one key each": lambda rng, hk, n: np.ones((hk, n), dtype=np.int64),
    "heads apart": lambda rng, hk, n: np.where(np.arange(hk)[:, None] == hk - 1, 20000, rng.integers(0, 5, (hk, n))),
}


@pytest.mark.parametrize("heads,batch", [(4, 12), (3, 20), (2, 65), (1, 130), (8, 33)])
@pytest.mark.parametrize("how", list(DEALT))
def test_chunks_dealt_out_by_the_lengths(how, heads, batch):
    """max_len is far above most lengths: the chunks follow the lengths.  One pool of few blocks serves all sequences."""
    rng = np.random.default_rng(900 + batch)
    lens = np.minimum(DEALT[how](rng, heads, batch), 20000)
    table = np.tile(rng.integers(0, 40, 20000 // 128 + 1).astype(np.int32), (batch, 1))
    for b in range(batch):
        table[b] = np.roll(table[b], b)
    pools = [Pool(1, 40, 128, heads) for _ in range(2)]
    for pool in pools:
        pool.codes[:] = rng.integers(0, 127, pool.codes.shape) + 128 * rng.integers(0, 2, pool.codes.shape)
        pool.byte[:] = rng.integers(112, 119, pool.byte.shape)
    q = queries(rng, batch, heads * 2, "bf16")
    out, lse, status = run(on_device(*pools, table), 0, q, [1] * batch, lens, "bf16", max_len=20000)
    assert status == 0
    some = sorted(set(rng.integers(0, batch, 6)) | {0, batch // 2, batch - 1})
    at = torch.tensor(some, device="cuda")
    check(out[at], lse[at], q[at], [1] * len(some), lens[:, some], *pools, table[some], 128, 0, parts_of("bf16", 1, 2))
    again, _, _ = run(on_device(*pools, table), 0, q, [1] * batch, lens, "bf16", max_len=20000)
    assert torch.equal(out, again)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_dealt_chunks_with_lengths_blocks_and_offsets_that_do_not_fit(dtype):
    rng = np.random.default_rng(950)
    lens = np.array([[9000, 20, 16000, 300, 7000, 50]]).repeat(4, 0)
    lens[1] = lens[1][::-1]
    k, v, table = build(rng, 4, lens[None], 128, width=400)
    ms, longest = [1, 2, 0, 1, 3, 1], 400 * 128
    q = queries(rng, sum(ms), 4, dtype)
    clean, clse, status = run(on_device(k, v, table), 0, q, ms, lens, dtype, max_len=longest)
    assert status == 0
    check(clean, clse, q, ms, lens, k, v, table, 128, 0, parts_of(dtype, 3, 1))
    bad, t2 = lens.copy(), table.copy()
    bad[0, 0], bad[2, 4] = longest + 1, -1
    t2[3, 1] = k.codes.shape[1]
    out, lse, status = run(on_device(k, v, t2), 0, q, ms, bad, dtype, max_len=longest)
    assert status == B.DEV_BAD_LENGTHS | B.DEV_BAD_BLOCK_TABLE
    row = {0: [0], 1: [1, 2], 3: [3], 4: [4, 5, 6], 5: [7]}
    gone = torch.zeros(sum(ms), 4, dtype=torch.bool, device="cuda")
    gone[row[0], 0] = True
    gone[row[4], 2] = True
    for h in range(4):                                       # the second block of sequence 3: heads that reach it
        gone[row[3], h] = bool(lens[h, 3] > 128)
    assert bool(torch.isnan(out[gone]).all()) and bool(torch.isfinite(out[~gone]).all())
    for h in range(4):
        bs_ = [b for b in (0, 1, 4, 5) if not ((b == 0 and h == 0) or (b == 4 and h == 2))]
        rows_ = [i for b in bs_ for i in row[b]]
        check(out[rows_][:, h:h + 1], lse[rows_][:, h:h + 1], q[rows_][:, h:h + 1], [ms[b] for b in bs_], lens[h:h + 1, bs_],
              _head(k, h), _head(v, h), table[bs_], 128, 0, parts_of(dtype, 3, 1))
    # offsets that descend: that sequence has no output, the others theirs
    off = np.concatenate([[0], np.cumsum(ms)]).astype(np.int32)
    off[2] = 0
    res = torch.full_like(q, 99.0)
    qs = B.Queries(q, res, _cuda(off), max_q=3, max_len=longest, scale=SCALE)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    qc = on_device(k, v, table)
    ws = torch.empty(B.skipkv_quant_attend_workspace_bytes(qc, qs) + 256, dtype=torch.uint8, device="cuda").fill_(0xFF)
    B.skipkv_quant_attend(qc, 0, qs, _cuda(lens.astype(np.int32)), ws, status)
    assert int(status.item()) == B.DEV_BAD_LENGTHS and bool((res[[4, 5, 6, 7]] != 99.0).all())


def _head(pool, h):
    one = Pool(1, pool.codes.shape[1], pool.codes.shape[2], 1)
    one.codes, one.byte = pool.codes[:, :, :, h:h + 1], pool.byte[:, h:h + 1]
    return one


@pytest.mark.parametrize("layout", ["slots", "heads"])
@pytest.mark.parametrize("batch,heads", [(1, 4), (40, 4), (3, 2)])
def test_one_and_many_sequences_in_both_layouts(layout, batch, heads):
    rng = np.random.default_rng(200 + batch)
    lens = rng.integers(1, 1200, (heads, batch))
    k, v, table = build(rng, heads, lens[None], 64)
    q = queries(rng, batch, heads * 4, "bf16")
    out, lse, status = run(on_device(k, v, table, heads_before_slots=layout == "heads"), 0, q, [1] * batch, lens, "bf16")
    assert status == 0
    check(out, lse, q, [1] * batch, lens, k, v, table, 64, 0, parts_of("bf16", 1, 4))


@pytest.mark.parametrize("longest", [2040, 2500, 6100])
@pytest.mark.parametrize("m,group", [(4, 4), (5, 4), (8, 4), (9, 4), (17, 1), (32, 1), (33, 1), (4, 8), (3, 7)])
def test_rows_around_the_change_of_kernel(m, group, longest):
    """16 and 17, 32 and 33 rows, below and above 2048 slots; the other sequence has fewer rows and keys."""
    rng = np.random.default_rng(300 + m)
    lens = np.array([[longest, 40], [longest // 3, 2]])
    k, v, table = build(rng, 2, lens[None], 32)
    ms = [m, 2]
    q = queries(rng, m + 2, 2 * group, "bf16")
    out, lse, status = run(on_device(k, v, table), 0, q, ms, lens, "bf16")
    assert status == 0
    check(out, lse, q, ms, lens, k, v, table, 32, 0, parts_of("bf16", m, group))


def test_many_rows_over_a_long_cache():
    """Two blocks of 256 rows, keys cut and joined, one head shorter than the queries."""
    rng = np.random.default_rng(400)
    lens = np.array([[9000], [130], [60]])
    k, v, table = build(rng, 3, lens[None], 128)
    q = queries(rng, 100, 12, "bf16")
    out, lse, status = run(on_device(k, v, table), 0, q, [100], lens, "bf16")
    assert status == 0
    check(out, lse, q, [100], lens, k, v, table, 128, 0, parts_of("bf16", 100, 4))
    assert bool((out[:40, 8:] == 0).all()) and bool((lse[:40, 8:] == -np.inf).all())


@pytest.mark.parametrize("ms,longest,width", [
    ([300, 1, 0, 500, 64], 1500, 12), ([0, 0, 700, 0, 0], 2600, 30), ([257] * 9, 900, 8), ([3] * 70 + [260], 300, 4), ([130, 260, 390], 40, 4)])
def test_many_rows_dealt_out(ms, longest, width):
    """More blocks of rows than half the CUs: whole turns first, the rest cut along the keys; sequences with few rows or none between."""
    rng = np.random.default_rng(410 + len(ms))
    heads, batch = 8, len(ms)
    lens = np.maximum(rng.integers(1, longest + 1, (heads, batch)), np.array(ms)[None, :] - 5)
    lens[2, 0], lens[3, batch - 1] = 0, max(longest, ms[-1])
    table = rng.integers(0, 40, (batch, width)).astype(np.int32)
    lens = np.minimum(lens, width * 128)
    pools = [Pool(1, 40, 128, heads) for _ in range(2)]
    for pool in pools:
        pool.codes[:] = rng.integers(0, 127, pool.codes.shape) + 128 * rng.integers(0, 2, pool.codes.shape)
        pool.byte[:] = rng.integers(112, 119, pool.byte.shape)
    q = queries(rng, sum(ms), heads * 4, "bf16")
    out, lse, status = run(on_device(*pools, table), 0, q, ms, lens, "bf16")
    assert status == 0
    check(out, lse, q, ms, lens, *pools, table, 128, 0, parts_of("bf16", max(ms), 4), heads=[0, 2, 3, 7])
    again, _, _ = run(on_device(*pools, table), 0, q, ms, lens, "bf16")
    assert torch.equal(out, again)
    # one head's length and one sequence's block that do not fit
    bad, t2 = lens.copy(), table.copy()
    bad[1, 0] = -1
    t2[batch - 1, 0] = 40
    got, gl, status = run(on_device(*pools, t2), 0, q, ms, bad, "bf16", max_len=int(lens.max()))
    gone = torch.zeros(out.shape[:2], dtype=torch.bool, device="cuda")
    gone[:ms[0], 4:8] = True
    for h in range(heads):
        if ms[-1] and lens[h, batch - 1] > 0:
            gone[sum(ms) - ms[-1]:, 4 * h:4 * h + 4] = True
    assert (status & B.DEV_BAD_LENGTHS != 0) == (ms[0] > 0) and (status & B.DEV_BAD_BLOCK_TABLE != 0) == (ms[-1] > 0)
    assert bool(torch.isnan(got[gone]).all()) and bool(torch.isfinite(got[~gone]).all())
    off = np.concatenate([[0], np.cumsum(ms)]).astype(np.int32)
    off[0] = -1
    qs = B.Queries(q, torch.zeros_like(q), _cuda(off), max_q=max(ms), max_len=int(lens.max()), scale=SCALE)
    qc, st = on_device(*pools, table), torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = torch.empty(B.skipkv_quant_attend_workspace_bytes(qc, qs) + 256, dtype=torch.uint8, device="cuda").fill_(0xFF)
    B.skipkv_quant_attend(qc, 0, qs, _cuda(lens.astype(np.int32)), ws, st)
    live = torch.isfinite(out)                                # (an output may be NaN or not; here none is)
    assert int(st.item()) == B.DEV_BAD_LENGTHS and bool(live.all()) and bool((qs.out[:ms[0]] == 0).all())
    if sum(ms) > ms[0]:
        check(qs.out[ms[0]:], None, q[ms[0]:], ms[1:], lens[:, 1:], *pools, table[1:], 128, 0, parts_of("bf16", max(ms), 4), heads=[5])


@pytest.mark.parametrize("heads,m,longest", [(3, 200, 9000), (1, 160, 300), (2, 900, 1500)])
def test_few_blocks_of_many_rows(heads, m, longest):
    """Blocks of 256 rows that are all cut alike and joined."""
    rng = np.random.default_rng(402 + m)
    lens = rng.integers(1, longest, (heads, 1))
    lens[0, 0] = longest
    k, v, table = build(rng, heads, lens[None], 32)
    q = queries(rng, m, 4 * heads, "bf16")
    out, lse, status = run(on_device(k, v, table), 0, q, [m], lens, "bf16")
    assert status == 0
    check(out, lse, q, [m], lens, k, v, table, 32, 0, parts_of("bf16", m, 4))
    table[0, longest // 32 - 1] = -7
    out, lse, status = run(on_device(k, v, table), 0, q, [m], lens, "bf16")
    assert status == B.DEV_BAD_BLOCK_TABLE and bool(torch.isnan(out[-1, :4]).all())
    out, lse, status = run(on_device(k, v, table), 0, q, [m], lens, "bf16", max_len=longest - 1)
    assert status & B.DEV_BAD_LENGTHS and bool(torch.isnan(out[:, :4]).all()) and bool(torch.isnan(lse[:, :4]).all())


@pytest.mark.parametrize("m,group,batch", [(200, 4, 2), (200, 4, 40), (60, 8, 2)])
def test_nan_values_reach_exactly_the_queries_that_see_them_in_blocks_of_many_rows(m, group, batch):
    """The blocks of rows differ in what they see, and so do the rows of one; NaN also in the middle of a cache and behind its end."""
    rng = np.random.default_rng(403 + batch)
    lens = rng.integers(m, 700, (1, batch))
    lens[0, :2] = 600, 450
    k, v, table = build(rng, 1, lens[None], 16)
    def poke(pool, b, t, d):
        pool.codes[0, table[b, t // 16], t % 16, 0, d] = 0xFF if d % 2 else 0x7F
    for d in (0, 5, 64, 127):
        poke(v, 0, 600 - 2, d)
        poke(v, 1, 450 - 1, d)
    poke(v, 1, 450 - m + 1, 3)                   # seen by all but the first
    poke(v, 1, 450 - m // 2, 70)                 # by query j where 450 - m + j >= 450 - m / 2: the second half
    poke(k, 0, 600 - 1, 9)
    poke(v, 0, 3, 77)
    q = queries(rng, batch * m, group, "bf16")
    out, lse, status = run(on_device(k, v, table), 0, q, [m] * batch, lens, "bf16")
    assert status == 0
    check(out[:2 * m], lse[:2 * m], q[:2 * m], [m, m], lens[:, :2], k, v, table[:2], 16, 0, parts_of("bf16", m, group))
    bad = torch.isnan(out).any(1).cpu().numpy()  # [tokens, D]
    assert bad[:m - 2].sum() == m - 2 and bad[m - 2].sum() == 5 and bad[m - 1].all()
    assert not bad[m].any() and bad[m + 1].sum() == 1 and bad[m + m // 2 - 1].sum() == 1 and bad[m + m // 2].sum() == 2
    assert bad[2 * m - 1].sum() == 6 and not bad[2 * m:].any()


@pytest.mark.parametrize("ms", [[70, 66, 80], [170, 166, 180]])
def test_many_rows_with_lengths_and_blocks_that_do_not_fit(ms):
    rng = np.random.default_rng(401)
    lens = np.array([[700, 300, 520], [80, 310, 90]])
    k, v, table = build(rng, 2, lens[None], 16)
    q = queries(rng, sum(ms), 8, "bf16")
    clean, _, _ = run(on_device(k, v, table), 0, q, ms, lens, "bf16")
    bad, t2 = lens.copy(), table.copy()
    bad[1, 0] = 701
    t2[2, 20] = k.codes.shape[1]                              # the first block id that does not exist; beyond head 1's keys
    out, lse, status = run(on_device(k, v, t2), 0, q, ms, bad, "bf16", max_len=700)
    assert status == B.DEV_BAD_LENGTHS | B.DEV_BAD_BLOCK_TABLE
    gone = torch.zeros(sum(ms), 8, dtype=torch.bool, device="cuda")
    gone[:ms[0], 4:] = True
    gone[ms[0] + ms[1]:, :4] = True
    assert bool(torch.isnan(out[gone]).all()) and bool(torch.isnan(lse[gone]).all()) and torch.equal(out[~gone], clean[~gone])


@pytest.mark.parametrize("m", [1, 5, 90, 200])
def test_in_a_graph_with_inputs_that_change(m):
    """Store, load and attention of one step, captured once and replayed with other lengths, rows and queries; eager work of the
    same kind in between."""
    rng = np.random.default_rng(500 + m)
    bs, heads, batch, cap = 16, 4, 3, 3200
    width = cap // bs
    table = rng.permutation(batch * width).reshape(batch, width).astype(np.int32)
    pools = [Pool(1, batch * width, bs, heads) for _ in range(2)]
    qc = on_device(*pools, table)
    off = _cuda(np.arange(batch + 1, dtype=np.int32) * m)
    full = _cuda(np.arange(batch + 1, dtype=np.int32) * cap)
    new = [torch.zeros((1, heads, batch * m, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    back = [torch.zeros((1, heads, batch * cap, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    rows = B.Cache(new[0], new[1], heads * 4, off, off, off, batch * m, 0)
    whole = B.Cache(back[0], back[1], heads * 4, full, full, full, batch * cap, 0)
    begin, end = (torch.zeros((1, heads, batch), dtype=torch.int32, device="cuda") for _ in range(2))
    q = torch.zeros((batch * m, heads * 4, D), dtype=torch.bfloat16, device="cuda")
    out = torch.zeros_like(q)
    qs = B.Queries(q, out, off, max_q=m, max_len=cap, scale=SCALE)
    ws = torch.empty(B.skipkv_quant_attend_workspace_bytes(qc, qs) + 256, dtype=torch.uint8, device="cuda")

    def step(stream=None):
        B.skipkv_quant_store(qc, rows, 0, begin, end, None, stream)
        B.skipkv_quant_attend(qc, 0, qs, end[0], ws, None, stream)
        B.skipkv_quant_load(qc, whole, 0, None, end, None, stream)

    def inputs(i):
        g = torch.Generator(device="cuda").manual_seed(i)
        for t in new + [q]:
            t.copy_(torch.randn(t.shape, generator=g, device="cuda"))
        n = torch.from_numpy(rng.integers(0, cap - m + 1, (1, heads, batch)).astype(np.int32))
        begin.copy_(n)
        end.copy_(n + m)
        for t in (qc.k, qc.v):                                 # finite codes of either sign
            t.copy_(torch.randint(0, 127, t.shape, generator=g, device="cuda", dtype=torch.uint8) + 128 * torch.randint(0, 2, t.shape, generator=g, device="cuda", dtype=torch.uint8))
        for t in (qc.k_exp, qc.v_exp):
            t.fill_(120)
        for t in back:
            t.zero_()
        out.zero_()

    inputs(0)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(1, 5):
        state = rng.bit_generator.state
        inputs(i)
        step()
        want = [t.clone() for t in (out, *back, qc.k, qc.v, qc.k_exp, qc.v_exp)]
        rng.bit_generator.state = state
        inputs(i)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, (out, *back, qc.k, qc.v, qc.k_exp, qc.v_exp)):
            assert torch.equal(a, b)
        assert bool(torch.isfinite(out).all()) and float(out.abs().max()) > 0


@pytest.mark.parametrize("batch,m,room", [(1, 1, 8192), (1, 8, 8192), (1, 300, 2048), (3, 100, 2048), (2, 1, 4096)])
def test_room_for_far_more_than_there_is(batch, m, room):
    """max_len is what a table row can hold, as a captured call has it; the lengths are a small part of it."""
    rng = np.random.default_rng(550 + batch)
    lens = rng.integers(m, 1200, (4, batch))
    k, v, table = build(rng, 4, lens[None], 16, width=room)
    q = queries(rng, batch * m, 16, "bf16")
    out, lse, status = run(on_device(k, v, table), 0, q, [m] * batch, lens, "bf16", max_len=16 * room)
    assert status == 0
    check(out, lse, q, [m] * batch, lens, k, v, table, 16, 0, parts_of("bf16", m, 4))


def test_two_calls_at_once_on_two_streams():
    rng = np.random.default_rng(600)
    lens = rng.integers(1, 3000, (4, 6))
    k, v, table = build(rng, 4, lens[None], 16)
    qc = on_device(k, v, table)
    cases = []
    for dtype, m in (("bf16", 1), ("bf16", 60), ("bf16", 200), ("bf16", 7), ("f32", 2)):
        ms, q = [m] * 6, queries(rng, 6 * m, 16, dtype)
        want, _, _ = run(qc, 0, q, ms, lens, dtype)
        out = torch.zeros_like(q)
        off = _cuda(np.arange(7, dtype=np.int32) * m)
        qs = B.Queries(q, out, off, max_q=m, max_len=int(lens.max()), scale=SCALE)
        ws = torch.empty(B.skipkv_quant_attend_workspace_bytes(qc, qs) + 256, dtype=torch.uint8, device="cuda")
        cases.append((qs, ws, want, torch.cuda.Stream()))
    n = _cuda(lens.astype(np.int32))
    torch.cuda.synchronize()
    for _ in range(5):
        for qs, ws, _, st in cases:
            B.skipkv_quant_attend(qc, 0, qs, n, ws, None, st)
    torch.cuda.synchronize()
    for qs, _, want, _ in cases:
        assert torch.equal(qs.out, want)


def test_sequences_that_share_blocks():
    """A common beginning held once: the same ids in two table rows, and one sequence twice in the batch."""
    rng = np.random.default_rng(700)
    lens = np.array([[200, 150, 200]])
    k, v, table = build(rng, 1, lens[None], 16)
    table[1, :5] = table[0, :5]
    table[2] = table[0]
    q = queries(rng, 3, 4, "bf16")
    q[2] = q[0]
    qc = on_device(k, v, table)
    out, lse, status = run(qc, 0, q, [1, 1, 1], lens, "bf16")
    assert status == 0 and torch.equal(out[2], out[0])
    check(out, lse, q, [1, 1, 1], lens, k, v, table, 16, 0, parts_of("bf16", 1, 4))
    off = _cuda(np.array([0, 200, 350, 550], dtype=np.int32))
    back = [torch.zeros((1, 1, 550, D), device="cuda") for _ in range(2)]
    B.skipkv_quant_load(qc, B.Cache(back[0], back[1], 4, off, off, off, 550, 0), 0, None, _cuda(lens[None].astype(np.int32)))
    for pool, t in ((k, back[0]), (v, back[1])):
        for b, at in enumerate((0, 200, 350)):
            n = int(lens[0, b])
            np.testing.assert_array_equal(t[0, 0, at:at + n].double().cpu().numpy(), pool.rows(0, 0, table[b], 16, n))


@pytest.mark.parametrize("byte", [0, 254, 255])
@pytest.mark.parametrize("dtype,m,group", [("bf16", 1, 4), ("f32", 2, 2), ("bf16", 40, 2), ("bf16", 12, 2), ("bf16", 200, 4)])
def test_scales_of_blocks_without_rows_do_not_matter(dtype, m, group, byte):
    """Every block that no sequence holds has a scale byte that no store writes and NaN codes; block 0 is one of them."""
    rng = np.random.default_rng(650)
    lens = np.array([[100, 65, 300], [47, 49, 1]])
    lens = np.maximum(lens, m)
    k, v, table = build(rng, 2, lens[None], 16)
    spare = next(p for p in range(k.codes.shape[1]) if p not in table)
    if spare != 0:                                            # move block 0 there
        for pool in (k, v):
            pool.codes[:, spare], pool.byte[:, :, spare] = pool.codes[:, 0], pool.byte[:, :, 0]
            pool.codes[:, 0] = 0x7F
        table = np.where(table == 0, spare, table)
    free = np.array([p for p in range(k.codes.shape[1]) if p not in table])
    for pool in (k, v):
        pool.byte[:, :, free] = byte
    q = queries(rng, 3 * m, 2 * group, dtype)
    out, lse, status = run(on_device(k, v, table), 0, q, [m] * 3, lens, dtype)
    assert status == 0
    check(out, lse, q, [m] * 3, lens, k, v, table, 16, 0, parts_of(dtype, m, group))


def test_what_the_binding_refuses(monkeypatch):
    rng = np.random.default_rng(800)
    lens = np.array([[20, 30]])
    k, v, table = build(rng, 1, lens[None], 16)
    qc = on_device(k, v, table)
    q = queries(rng, 2, 4, "bf16")
    off = _cuda(np.array([0, 1, 2], dtype=np.int32))
    n = _cuda(lens.astype(np.int32))
    qs = B.Queries(q, torch.zeros_like(q), off, max_q=1, max_len=30, scale=SCALE)
    rows = B.Cache(*(torch.zeros((1, 1, 2, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)), 4, off, off, off, 2, 0)
    pages = B.Pages(qc.block_table, _cuda(np.array([2, 2], dtype=np.int32)), torch.zeros(9, dtype=torch.int32, device="cuda"),
                    torch.zeros(1, dtype=torch.int32, device="cuda"), 16)
    ws = torch.empty(4096, dtype=torch.uint8, device="cuda")
    for bad in (n.long(), n.cpu(), n[:, :1], torch.stack([n, n], 2)[:, :, 0]):
        with pytest.raises(AssertionError):
            B.skipkv_quant_attend(qc, 0, qs, bad, ws)
    for bad in (n[None].long(), n[None].cpu(), n[None, :, :1]):
        for call in (B.skipkv_quant_store, B.skipkv_quant_load):
            with pytest.raises(AssertionError):
                call(qc, rows, 0, bad, None)
            with pytest.raises(AssertionError):
                call(qc, rows, 0, None, bad)
    for bad in (dict(q_off=off.long()), dict(q_off=off.cpu()), dict(q_off=off[:2]), dict(out=torch.zeros_like(q).float()), dict(out=qs.out.cpu()),
                dict(lse=torch.zeros(2, 3, device="cuda"))):
        d = dict(q=q, out=qs.out, q_off=off, max_q=1, max_len=30, scale=SCALE)
        with pytest.raises(AssertionError):
            B.skipkv_quant_attend(qc, 0, B.Queries(**dict(d, **bad)), n, ws)
    with pytest.raises(AssertionError):
        B.skipkv_pages_update(pages, n.long(), off, 2, None, ws)
    with pytest.raises(AssertionError):
        B.skipkv_pages_update(pages, n, off, 2, torch.zeros(3, dtype=torch.int32, device="cuda"), ws)
    with pytest.raises(AssertionError):
        B.skipkv_pages_update(pages, n, off[:2], 1, None, ws)
    with pytest.raises(B.SkipKVError):
        B.skipkv_pages_update(pages, n, off, 2, None, ws[:16])
    # another current device than the tensors'
    here = torch._C._cuda_getDevice()
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: here + 1)
    for call in (lambda: B.skipkv_quant_attend(qc, 0, qs, n, ws), lambda: B.skipkv_quant_store(qc, rows, 0, None, None),
                 lambda: B.skipkv_quant_load(qc, rows, 0, None, None), lambda: B.skipkv_pages_update(pages, n, off, 2, None, ws)):
        with pytest.raises(AssertionError, match="another device"):
            call()
