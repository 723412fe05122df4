"""The blocks' book where a table or a count is damaged: what the calls count, and
that one request never comes to name another's block.  Against the plain-loop
oracle (oracle/blocks.py), every table, count, free list and cache byte."""
import pytest

from test_gpu_blocks import Pair

pytestmark = pytest.mark.gpu


def _set(p, row, at, value):
    p.pool.table[row, at] = p.book.table[row, at] = value


@pytest.mark.parametrize("entry", [-1, 50, -7])
def test_a_fork_inside_a_block_that_the_parent_lacks(entry):
    """No block to copy: the child has none there, nothing is taken, and it counts.
    Beside forks that are in order, and one that ends with a whole block."""
    p = Pair(50, 32, 4, 8, 5)
    p.extend([0, 1], [18, 7])
    _set(p, 0, 2, entry)
    before, free = p.book.errors, len(p.book.free)
    p.fork([0, 1, 0], [2, 3, 4], [10, 7, 8])
    assert p.book.errors == before + 1 and len(p.book.free) == free - 1
    assert p.book.table[2].tolist()[2:] == [-1, -1, -1]
    # among the whole blocks: none is shared as none, an id that is none counts
    p.fork([0], [5], [16])
    assert p.book.errors == before + (1 if entry == -1 else 2)


@pytest.mark.parametrize("blocks", [30, 3000, 40000])
def test_entries_that_name_free_blocks_do_not_survive_a_compaction(blocks):
    """Free ids below the live count, into which live blocks move, and free ids past it."""
    p = Pair(blocks, 16, 1, 6, 10)
    p.extend([0, 1, 2], [10, 5, 8])                  # ids 0 .. 22
    p.free([0])                                      # 0 .. 9 are free; 13 are live, so 10 to 12 stay
    for at, entry in enumerate((2, 9, blocks - 1, 12, blocks, -5)):
        _set(p, 3, at, entry)
    p.book.ref[12] += 1                              # a second entry for a live block is no damage
    p.pool.ref_count[12] += 1
    before = p.book.errors
    p.compact()
    assert p.book.errors == before + 5               # three free, two that are none
    assert p.book.table[3].tolist() == [-1, -1, -1, 12, blocks, -5] + [-1] * 4
