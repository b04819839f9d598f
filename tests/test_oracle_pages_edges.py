"""Pins of the oracle's pool where its table names blocks that no count stands for."""
import numpy as np

from oracle import pages


def test_a_fork_does_not_share_what_is_free():
    p = pages.Pool(10, 6, 4, np.arange(10).reshape(1, 10, 1).copy())
    p.reserve([0, 1], [36, 64])                            # blocks 0, 1, 2 and 3 .. 6
    p.table[0, 0], p.table[1, 1], p.table[1, 2] = 7, 9, 10   # free; free; none of the pool
    p.fork([0, 1], [2, 3])                                 # the copy of block 2 goes to 7, which row 0 names by mistake
    assert p.problems == {"invalid"} and p.lens.tolist() == [36, 64, 36, 64, 0, 0]
    assert p.table[2].tolist() == [-1, 1, 7, -1] and p.table[3].tolist() == [3, -1, -1, 6]
    assert p.refs.tolist() == [1, 2, 1, 2, 1, 1, 2, 1, 0, 0] and p.contents[0, 7, 0] == 2


def test_a_fork_without_its_partly_filled_block_is_refused():
    for entry in (-1, 7, 10):
        p = pages.Pool(10, 6, 4, np.zeros((0, 10, 1)))
        p.reserve([0, 1], [36, 20])
        p.table[0, 2] = entry
        refs = p.refs.copy()
        p.fork([0], [2])
        assert p.problems == {"invalid"} and p.lens[2] == 0 and p.table[2].tolist() == [-1] * 4 and np.array_equal(p.refs, refs)
        p.fork([0, 1], [2, 3])                             # the one behind it is served
        assert p.lens.tolist() == [36, 20, 0, 20, 0, 0] and p.table[3].tolist() == [3, 5, -1, -1]
