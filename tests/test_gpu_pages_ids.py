"""Block ids that do not exist, in the tables and on the stack of free blocks: no slot is made of one, and they are reported."""
import numpy as np
import pytest
import torch

from paper_2512_07993_amd import binding as B

from test_gpu_pages import _check, _state, _update, plain

pytestmark = pytest.mark.gpu
BS = 16


def _expect(state, lens, counts):
    """The plain form, whose slots in blocks that do not exist are -1; status: ids that were moved or made slots of."""
    table, held, free, n_free, slots, status = plain(*state, BS, lens, counts)
    n_blocks = len(free)
    was_held, was_free = state[1], state[3]
    off = np.concatenate([[0], np.cumsum(counts)]).astype(int)
    bad = False
    for b in range(len(held)):
        bad |= any(not 0 <= x < n_blocks for x in table[b, was_held[b]:held[b]])                   # taken
        for r in range(lens.shape[0]):
            for i in range(off[b], off[b + 1]):
                pos = int(lens[r, b]) + i - off[b]
                if pos // BS < held[b] and not 0 <= table[b, pos // BS] < n_blocks:
                    slots[r, i] = -1
                    bad = True
    bad |= any(not 0 <= x < n_blocks for x in free[was_free:n_free])                               # given back and still there
    return table, held, free, n_free, slots, status | (B.DEV_BAD_BLOCK_TABLE if bad else 0)


def _same(state, lens, counts):
    pg, slots, status = _update(state, BS, lens, counts)
    table, held, free, n_free, want, bits = _expect(state, lens, counts)
    np.testing.assert_array_equal(pg.block_table.cpu().numpy(), table)
    np.testing.assert_array_equal(pg.n_held.cpu().numpy(), held)
    np.testing.assert_array_equal(pg.free_list.cpu().numpy(), free)
    assert int(pg.n_free.item()) == n_free
    np.testing.assert_array_equal(slots.cpu().numpy(), want)
    assert status == bits
    return slots, status


IDS = [-1, -2 ** 31, 2 ** 31 - 1, "n_blocks"]


@pytest.mark.parametrize("rows", [1, 9])
@pytest.mark.parametrize("bad", IDS)
def test_an_id_that_a_sequence_holds(bad, rows):
    rng = np.random.default_rng(40)
    for entry in (0, 1, 2):
        state = _state(rng, 3, 8, [2, 3, 1], 9)
        state[0][1, entry] = len(state[2]) if bad == "n_blocks" else bad
        lens = np.tile(np.array([[20, 33, 5]]), (rows, 1))                # the new tokens of sequence 1: entries 2 and 3
        slots, status = _same(state, lens, [1, 20, 0])
        assert (status != 0) == (entry == 2) and bool(((slots[:, 1:21] < 0).sum(1) == (15 if entry == 2 else 0)).all()) and bool((slots[:, 0] >= 0).all())


@pytest.mark.parametrize("bad", IDS)
def test_an_id_that_is_given_back(bad):
    """It goes where the others go - onto the stack or to a sequence that grows - and is reported in both cases."""
    rng = np.random.default_rng(41)
    for counts in ([0, 0, 0], [0, 0, 40]):
        state = _state(rng, 3, 8, [2, 5, 1], 9)
        state[0][1, 4] = len(state[2]) if bad == "n_blocks" else bad
        _, status = _same(state, np.array([[20, 40, 5]]), counts)
        assert status == B.DEV_BAD_BLOCK_TABLE


@pytest.mark.parametrize("bad", IDS)
def test_an_id_on_the_stack(bad):
    rng = np.random.default_rng(42)
    for depth, seen in ((1, True), (2, True), (3, False)):                 # two blocks are taken
        state = _state(rng, 3, 8, [2, 2, 1], 9)
        state[2][state[3] - depth] = len(state[2]) if bad == "n_blocks" else bad
        _, status = _same(state, np.array([[20, 20, 5]]), [0, 20, 20])
        assert status == (B.DEV_BAD_BLOCK_TABLE if seen else 0)


def test_ids_that_exist_are_not_reported():
    """The first and the last block, in every role."""
    rng = np.random.default_rng(43)
    for trial in range(4):
        state = _state(rng, 4, 8, [2, 5, 1, 0], 4)
        _check(state, BS, np.array([[20, 3, 5, 0]]), [10, 1, 40, 17])
