"""Pools whose tables name blocks that no count stands for: what every call does with such an entry is the oracle's, whatever the
order in which the device gets to it."""
import numpy as np
import pytest
import torch

from paper_2602_09323_b200 import binding
from tests.test_gpu_pages import Both, ints

pytestmark = pytest.mark.gpu


def stale(p, row, j, block):
    p.pages.block_table[row, j] = block
    p.ref.table[row, j] = block


@pytest.mark.parametrize("blocks", [300, 32768, 32769, 100000])
def test_a_fork_of_a_table_that_names_free_blocks(blocks):
    """Entries of free blocks among full ones, one of them the very block that the call hands out: none is shared, and the
    blocks handed out are those of the counts before the call."""
    p = Both(blocks, 40, 12, layers=2, hkv=1, seed=101)
    p.reserve(list(range(8)), [190, 33, 17, 64, 100, 5, 48, 130])
    free = np.nonzero(p.ref.refs == 0)[0]
    stale(p, 0, 3, int(free[0]))                           # the block that the first copy gets
    stale(p, 0, 4, int(free[1]))
    stale(p, 3, 0, int(free[2]))
    stale(p, 4, 2, blocks)                                 # none of the pool
    stale(p, 7, 5, blocks - 1)
    p.fork([0, 1, 2, 3, 4, 5, 6, 7, 0, 7], list(range(10, 20)))
    p.check("full blocks")
    assert p.ref.lens[10:20].tolist() == [190, 33, 17, 64, 100, 5, 48, 130, 190, 130]
    # the counts are those of the entries that name a block
    names = p.ref.table[8:][p.ref.table[8:] >= 0]
    assert np.all(p.ref.refs[names] > 0)
    p.release([10, 18])
    p.release([13, 14, 17, 19])
    p.check("released again")


@pytest.mark.parametrize("blocks", [300, 40000])
def test_a_fork_whose_partly_filled_block_is_not_in_use_is_refused(blocks):
    p = Both(blocks, 20, 6, layers=1, hkv=2, dim=128, seed=103)
    p.reserve([0, 1, 2, 3, 4], [20, 40, 70, 33, 32])
    stale(p, 0, 1, -1)
    stale(p, 1, 2, blocks)
    stale(p, 2, 4, int(np.nonzero(p.ref.refs == 0)[0][0]))
    p.fork([0, 1, 2, 3, 4, 2], [10, 11, 12, 13, 14, 15])
    assert p.ref.problems == {"invalid"} and p.ref.lens[10:16].tolist() == [0, 0, 0, 33, 32, 0]
    p.check("three refused")
    p.fork([3, 13], [10, 11])
    p.check("nothing wrong")
    assert not p.ref.problems


def test_a_fork_with_stale_entries_many_times_over():
    """The same call on the same pool gives the same result, with as many CTAs at work as there are SMs."""
    rows, width = 600, 96
    for blocks in (32768, 33000):
        rng = np.random.default_rng(blocks)
        p = Both(blocks, rows, width, layers=1, hkv=1, seed=107)
        p.reserve(list(range(100)), [int(x) for x in rng.integers(1, 16 * width, 100)])
        free = np.nonzero(p.ref.refs == 0)[0]
        for k in range(300):                               # the blocks that the call will hand out, as full entries of parents
            row = int(rng.integers(0, 100))
            if p.ref.lens[row] >= 32:
                stale(p, row, int(rng.integers(0, p.ref.lens[row] // 16)), int(free[k]))
        kids = list(range(100, 600))
        parents = [int(x) for x in rng.integers(0, 100, 500)]
        first = [x.clone() for x in (p.pages.refs, p.pages.block_table, p.pages.context_lens)]
        p.fork(parents, kids)
        p.check("once")
        for turn in range(5):
            for x, y in zip((p.pages.refs, p.pages.block_table, p.pages.context_lens), first):
                x.copy_(y)
            binding.pages_fork(p.set, p.pages, ints(parents), ints(kids), p.ws)
            torch.cuda.synchronize()
            assert np.array_equal(p.pages.refs.cpu().numpy(), p.ref.refs), turn
            assert np.array_equal(p.pages.block_table.cpu().numpy(), p.ref.table), turn
            assert np.array_equal(p.pages.context_lens.cpu().numpy(), p.ref.lens), turn
            assert binding.workspace_status(p.ws) == -1
            binding.workspace_init(p.ws)


def test_room_taken_ahead_of_what_is_written():
    """The length set back to the tokens written: a windowed release keeps what the next query sees, a fork shares what is written, and
    the room stays with its row."""
    p = Both(60, 8, 12, layers=1, seed=109)

    def reserve_and_set_back(rows, room, written):
        p.reserve(rows, room)
        p.pages.context_lens[torch.tensor(rows, device="cuda")] = ints(written)
        p.ref.lens[rows] = written

    reserve_and_set_back([0, 1], [180, 100], [100, 33])
    table = p.ref.table.copy()
    p.release([0, 1], 40, 3)                              # by 180 and 100 tokens the blocks of tokens 48..63, and of 16..47, would go too
    p.check("windowed release")
    assert p.ref.table[0].tolist() == [table[0, 0], -1, -1] + table[0, 3:].tolist() and p.ref.table[1].tolist() == table[1].tolist()
    p.fork([0, 1], [4, 5])
    p.check("fork")
    assert p.ref.lens.tolist() == [100, 33, 0, 0, 100, 33, 0, 0] and p.ref.table[5, 3] == -1
    free = int(np.sum(p.ref.refs == 0))
    reserve_and_set_back([0, 1, 4], [180, 110, 113], [101, 34, 101])
    p.check("more of what is there already")
    assert int(np.sum(p.ref.refs == 0)) == free - 1       # the child's eighth block; the others had theirs
    p.release([0, 1, 4, 5])
    p.check("all of it")
    assert not p.ref.refs.any()
