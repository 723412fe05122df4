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
