"""Block tables, the stack of free blocks and the slots of new tokens against a plain sequential form."""
import numpy as np
import pytest
import torch

from paper_2512_07993_amd import binding as B

pytestmark = pytest.mark.gpu


def plain(table, held, free, n_free, bs, lens, counts):
    """In order of the sequences: first everything is given back, then blocks are taken off the top."""
    table, held, free = table.copy(), held.copy(), free.copy()
    stack = list(free[:n_free])
    batch, stride = table.shape
    need = [-(-(int(lens[:, b].max()) + counts[b]) // bs) for b in range(batch)]
    status = 0
    for b in range(batch):
        if need[b] > stride:
            status |= B.DEV_OUT_OF_BLOCKS
        elif need[b] < held[b]:
            stack += list(table[b, need[b]:held[b]])
            held[b] = need[b]
    low = n_free                       # entries below this were never popped
    refused = False
    for b in range(batch):
        grow = need[b] - held[b]
        if need[b] > stride or grow <= 0:
            continue
        refused = refused or grow > len(stack)
        if refused:
            status |= B.DEV_OUT_OF_BLOCKS
            continue
        for i in range(grow):
            table[b, held[b] + i] = stack.pop()
        held[b] = need[b]
    free[low:len(stack)] = stack[low:]
    slots = np.full((lens.shape[0], int(sum(counts))), -1, dtype=np.int32)
    at = 0
    for b in range(batch):
        for i in range(counts[b]):
            for r in range(lens.shape[0]):
                pos = int(lens[r, b]) + i
                if pos // bs < held[b]:
                    slots[r, at + i] = table[b, pos // bs] * bs + pos % bs
        at += counts[b]
    return table, held, free, len(stack), slots, status


def _state(rng, batch, stride, held, spare):
    blocks = int(np.sum(held)) + spare + 1
    perm = rng.permutation(blocks).astype(np.int32)
    table = np.full((batch, stride), -9, dtype=np.int32)
    at = 0
    for b in range(batch):
        table[b, :held[b]] = perm[at:at + held[b]]
        at += held[b]
    free = np.full(blocks, -5, dtype=np.int32)
    free[:blocks - at] = perm[at:]
    return table, np.asarray(held, dtype=np.int32), free, blocks - at


def _cuda(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def _update(state, bs, lens, counts, wide=0):
    table, held, free, n_free = state
    big = torch.full((table.shape[0], table.shape[1] + wide), -3, dtype=torch.int32, device="cuda")
    big[:, :table.shape[1]] = _cuda(table)
    pg = B.Pages(big[:, :table.shape[1]] if wide == 0 else big, _cuda(held), _cuda(free), _cuda(np.array([n_free], dtype=np.int32)), bs)
    off = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    slots = torch.full((lens.shape[0], int(off[-1])), -77, dtype=torch.int32, device="cuda")
    ws = torch.empty(B.skipkv_pages_workspace_bytes(pg) + 256, dtype=torch.uint8, device="cuda").fill_(0xAB)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.skipkv_pages_update(pg, _cuda(lens.astype(np.int32)), _cuda(off), int(off[-1]), slots, ws, status)
    torch.cuda.synchronize()
    return pg, slots, int(status.item())


def _check(state, bs, lens, counts):
    pg, slots, status = _update(state, bs, lens, counts)
    table, held, free, n_free, want, bits = plain(*state, bs, lens, counts)
    np.testing.assert_array_equal(pg.block_table.cpu().numpy(), table)
    np.testing.assert_array_equal(pg.n_held.cpu().numpy(), held)
    assert int(pg.n_free.item()) == n_free
    np.testing.assert_array_equal(pg.free_list.cpu().numpy(), free)
    np.testing.assert_array_equal(slots.cpu().numpy(), want)
    assert status == bits
    # no block is held twice or lost
    have = [x for b in range(len(held)) for x in table[b, :held[b]]] + list(free[:n_free])
    assert sorted(have) == sorted(set(have)) and len(have) == len(state[2])
    return pg


@pytest.mark.parametrize("batch,rows,bs,spare", [(1, 1, 16, 3), (5, 1, 1, 40), (17, 6, 16, 30), (64, 112, 16, 200), (300, 3, 32, 100), (257, 2, 7, 2000)])
def test_tables_follow_the_lengths(batch, rows, bs, spare):
    rng = np.random.default_rng(batch * 7 + rows)
    for trial in range(3):
        held = rng.integers(0, 40, batch)
        base = rng.integers(0, 36 * bs, batch) if trial < 2 else held * bs
        lens = np.maximum(base[None, :] - rng.integers(0, 2 * bs + 1, (rows, batch)), 0)
        counts = [int(x) for x in rng.integers(0, 3 if trial == 2 else 4 * bs, batch)]
        _check(_state(rng, batch, 48, held, spare), bs, lens, counts)


def test_the_first_sequence_that_does_not_fit_ends_the_growth():
    rng = np.random.default_rng(2)
    held = [2, 3, 1, 5, 0]
    lens = np.array([[3 * 16, 3 * 16, 6 * 16, 2 * 16, 16]])              # grow by 1, 0, 5; give back 3; grow by 1
    for spare in (-1, 0, 1, 2, 3, 4):
        state = _state(rng, 5, 8, held, spare)
        _check(state, 16, lens, [0, 0, 0, 0, 0])
        _check(state, 16, lens, [1, 0, 3, 0, 16])


def test_a_row_that_is_too_short_leaves_its_sequence_alone():
    rng = np.random.default_rng(3)
    state = _state(rng, 3, 6, [6, 2, 2], 10)
    _check(state, 16, np.array([[96, 40, 1]]), [1, 2, 3])                # 97 tokens need 7 entries of 6


def test_all_sequences_leave_and_come_back():
    rng = np.random.default_rng(4)
    state = _state(rng, 9, 20, [7] * 9, 5)
    pg = _check(state, 16, np.zeros((4, 9), dtype=np.int64), [0] * 9)
    state = (pg.block_table.cpu().numpy(), pg.n_held.cpu().numpy(), pg.free_list.cpu().numpy(), int(pg.n_free.item()))
    assert state[3] == 69 and state[1].sum() == 0
    _check(state, 16, np.zeros((4, 9), dtype=np.int64), [100] * 9)


def test_the_largest_batch_and_no_new_tokens():
    rng = np.random.default_rng(5)
    held = rng.integers(0, 3, 4096)
    state = _state(rng, 4096, 4, held, 4096)
    _check(state, 16, rng.integers(0, 60, (1, 4096)), [0] * 4096)
    _check(state, 16, rng.integers(0, 60, (2, 4096)), [int(x) for x in rng.integers(0, 2, 4096)])


def test_table_rows_may_lie_further_apart():
    rng = np.random.default_rng(6)
    state = _state(rng, 3, 5, [1, 4, 2], 9)
    lens, counts = np.array([[30, 20, 64]]), [5, 0, 1]
    pg, slots, status = _update(state, 16, lens, counts, wide=3)
    table, held, free, n_free, want, bits = plain(*state, 16, lens, counts)
    np.testing.assert_array_equal(pg.block_table.cpu().numpy()[:, :5], table)
    assert bool((pg.block_table[:, 5:] == -3).all()) and status == bits == 0
    np.testing.assert_array_equal(slots.cpu().numpy(), want)


def test_lengths_and_counts_that_cannot_be():
    rng = np.random.default_rng(7)
    state = _state(rng, 3, 8, [2, 2, 2], 9)
    lens = np.array([[20, -1, 40], [20, 5, 40]])
    pg, slots, status = _update(state, 16, lens, [1, 1, 1])
    assert status == B.DEV_BAD_LENGTHS
    assert pg.n_held.tolist() == [2, 2, 3] and bool((slots[:, 1] == -1).all()) and int((slots[:, [0, 2]] < 0).sum()) == 0
    # counts that descend
    off = torch.tensor([0, 5, 3, 6], dtype=torch.int32, device="cuda")
    pg, _, _ = _update(state, 16, np.array([[20, 20, 20]]), [0, 0, 0])
    before = pg.n_held.clone()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = torch.empty(4096, dtype=torch.uint8, device="cuda")
    slots = torch.zeros((1, 6), dtype=torch.int32, device="cuda")
    B.skipkv_pages_update(pg, torch.full((1, 3), 20, dtype=torch.int32, device="cuda"), off, 6, slots, ws, status)
    assert int(status.item()) == B.DEV_BAD_LENGTHS and pg.n_held[1] == before[1]


@pytest.mark.parametrize("what", ["held", "negative", "free", "overflow"])
def test_a_state_that_cannot_be_is_left_as_it_is(what):
    rng = np.random.default_rng(8)
    table, held, free, n_free = _state(rng, 3, 8, [2, 3, 2], 4)
    if what == "held":
        held[1] = 9
    elif what == "negative":
        held[1] = -1
    elif what == "free":
        n_free = len(free) + 1
    else:
        n_free = len(free) - 1                                          # what sequence 1 gives back does not fit
    pg, slots, status = _update((table, held, free, n_free), 16, np.array([[20, 1, 20]]), [1, 1, 1])
    assert status == B.DEV_BAD_BLOCK_TABLE
    np.testing.assert_array_equal(pg.block_table.cpu().numpy(), table)
    np.testing.assert_array_equal(pg.n_held.cpu().numpy(), held)
    np.testing.assert_array_equal(pg.free_list.cpu().numpy(), free)
    assert int(pg.n_free.item()) == n_free and bool((slots == -1).all())


def test_without_a_slot_map_or_new_tokens():
    rng = np.random.default_rng(9)
    state = _state(rng, 2, 8, [4, 1], 3)
    table, held, free, n_free = state
    pg = B.Pages(_cuda(table), _cuda(held), _cuda(free), _cuda(np.array([n_free], dtype=np.int32)), 16)
    ws = torch.empty(4096, dtype=torch.uint8, device="cuda")
    B.skipkv_pages_update(pg, torch.tensor([[10, 50]], dtype=torch.int32, device="cuda"), None, 0, None, ws)
    want = plain(*state, 16, np.array([[10, 50]]), [0, 0])
    np.testing.assert_array_equal(pg.block_table.cpu().numpy(), want[0])
    assert pg.n_held.tolist() == [1, 4] and int(pg.n_free.item()) == want[3]


@pytest.mark.parametrize("bs", [1, 3, 7, 16, 100, 128, 1000])
def test_many_new_tokens_at_every_block_size(bs):
    """Tokens of a sequence that span several workgroups, empty sequences between them, blocks of sizes that no shift divides."""
    rng = np.random.default_rng(30 + bs)
    batch, rows = 9, 11
    lens = rng.integers(0, 700, (rows, batch))
    lens[:, 3] = 0
    counts = [1, 0, 700, 257, 0, 0, 255, 1, 300]
    need = [-(-(int(lens[:, b].max()) + counts[b]) // bs) for b in range(batch)]
    held = [max(0, need[b] + (-1) ** b * int(rng.integers(0, 5))) for b in range(batch)]
    state = _state(rng, batch, max(need) + 5, held, 40)
    _check(state, bs, lens, counts)


def test_more_rows_than_a_thread_takes_at_a_time():
    rng = np.random.default_rng(31)
    state = _state(rng, 300, 6, rng.integers(0, 7, 300), 700)
    lens = rng.integers(0, 80, (97, 300))
    _check(state, 16, lens, [int(x) for x in rng.integers(0, 4, 300)])


def test_offsets_below_zero_and_tokens_of_nobody():
    """A first offset below zero and a total beyond the last offset: slots of -1 and nothing else."""
    rng = np.random.default_rng(32)
    table, held, free, n_free = _state(rng, 2, 8, [2, 2], 9)
    pg = B.Pages(_cuda(table), _cuda(held), _cuda(free), _cuda(np.array([n_free], dtype=np.int32)), 16)
    off = torch.tensor([-2 ** 31, 2, 4], dtype=torch.int32, device="cuda")
    slots = torch.full((1, 6), -7, dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = torch.empty(4096, dtype=torch.uint8, device="cuda")
    B.skipkv_pages_update(pg, torch.tensor([[20, 20]], dtype=torch.int32, device="cuda"), off, 6, slots, ws, status)
    t = pg.block_table.cpu().numpy()
    assert slots.tolist() == [[-1, -1, int(t[1, 1]) * 16 + 4, int(t[1, 1]) * 16 + 5, -1, -1]]
    assert pg.n_held.tolist() == [2, 2] and int(status.item()) == B.DEV_OUT_OF_BLOCKS
