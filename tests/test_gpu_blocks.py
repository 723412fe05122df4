"""The block cache's bookkeeping against the plain-loop oracle (oracle/blocks.py):
every table, count, free list and cache byte, after every call."""
import numpy as np
import pytest
import torch

from oracle.blocks import Book
from paper_2609_15030_amd import api
from paper_2609_15030_amd import linattn as la

pytestmark = pytest.mark.gpu


def _i32(x):
    return torch.tensor(list(x), dtype=torch.int32, device="cuda")


class Pair:
    """A pool on the device and its oracle, compared after every step."""

    def __init__(self, blocks, block_bytes, bt, rows, width, seed=1):
        self.pool = api.BlockPool.new(blocks, block_bytes, bt, rows, width)
        rng = np.random.default_rng(seed)
        cache = rng.integers(0, 256, (blocks, block_bytes), dtype=np.uint8)
        self.pool.cache.copy_(torch.from_numpy(cache))
        self.book = Book(cache, bt, np.full((rows, width), -1, np.int32), np.zeros(blocks, np.int32),
                         range(blocks - 1, -1, -1))

    def same(self, what):
        torch.cuda.synchronize()
        p, b = self.pool, self.book
        assert np.array_equal(p.table.cpu().numpy(), b.table), what
        assert np.array_equal(p.ref_count.cpu().numpy(), b.ref), what
        n = int(p.free_count)
        assert n == len(b.free) and p.free_list[:n].tolist() == b.free, what
        assert int(p.err_count) == b.errors, what
        assert np.array_equal(p.cache.cpu().numpy(), b.cache), what

    def extend(self, rows, lens):
        self.pool.extend(_i32(rows), _i32(lens))
        self.book.extend(rows, lens)
        self.same(("extend", rows, lens))

    def fork(self, parents, children, lens):
        self.pool.fork(_i32(parents), _i32(children), _i32(lens))
        self.book.fork(parents, children, lens)
        self.same(("fork", parents, children, lens))

    def free(self, rows):
        self.pool.free(_i32(rows))
        self.book.release(rows)
        self.same(("free", rows))

    def compact(self):
        new = torch.full((len(self.book.ref),), 7, dtype=torch.int32, device="cuda")
        self.pool.compact(new)
        want = self.book.compact()
        self.same("compact")
        assert np.array_equal(new.cpu().numpy(), want)

    def copy(self, src, dst):
        self.pool.copy(_i32(src), _i32(dst))
        self.book.copy(src, dst)
        self.same(("copy", src, dst))


def test_a_life_of_a_pool():
    p = Pair(40, 48, 16, 8, 6)
    p.extend([0, 1, 2], [96, 17, 0])
    p.extend([0, 1], [96, 50])                       # grown rows keep their blocks
    p.fork([0, 0, 1, 1], [3, 4, 5, 6], [96, 33, 16, 50])
    p.extend([4, 6], [60, 64])
    p.free([0])                                      # its shared blocks stay
    p.compact()
    p.free([3, 5])
    p.copy([int(p.book.table[1, 0]), -1], [39, 5])
    p.compact()
    p.fork([6], [0], [49])
    p.free([0, 1, 2, 4, 6, 7])
    assert len(p.book.free) == 40
    p.compact()


def test_a_pool_that_runs_out():
    p = Pair(5, 16, 4, 4, 4)
    p.extend([0, 1], [16, 16])                       # eight wanted, five there
    p.fork([0, 1], [2, 3], [6, 3])                   # none left for the copies
    p.free([1, 0])
    p.free([2, 3])
    p.extend([2], [16])


@pytest.mark.parametrize("seed", range(3))
def test_random_calls(seed):
    rng = np.random.default_rng(seed)
    bt, width, rows = 8, 9, 12
    p = Pair(60, 32 + 16 * seed, bt, rows, width, seed)
    for _ in range(25):
        what = rng.integers(0, 5)
        used = [r for r in range(rows) if (p.book.table[r] >= 0).any()]
        empty = [r for r in range(rows) if r not in used]
        if what <= 1:
            pick = rng.permutation(rows)[:rng.integers(1, 4)].tolist()
            p.extend(pick, rng.integers(0, bt * width + 1, len(pick)).tolist())
        elif what == 2 and used and empty:
            n = int(rng.integers(1, min(len(empty), 3) + 1))
            par = rng.choice(used, n).tolist()
            p.fork(par, empty[:n], [int(rng.integers(0, bt * int((p.book.table[r] >= 0).sum()) + 1)) for r in par])
        elif what == 3 and used:
            p.free(rng.permutation(used)[:rng.integers(1, 3)].tolist())
        else:
            p.compact()


def test_bad_ids_are_counted():
    p = Pair(12, 16, 4, 4, 3)
    p.extend([0, 9, -1, 1], [8, 4, 4, 13])           # two rows that are none, a length past the table
    p.fork([0, 7, 0, 2], [2, 3, -3, 2], [8, 4, 4, 4])
    p.fork([0], [3], [99])
    p.copy([0, 12, 3], [5, 6, -2])
    p.free([8, 0])
    # an entry that names no block, and a reference taken back twice
    p.pool.table[1, 0] = 77
    p.book.table[1, 0] = 77
    p.pool.table[0, 0] = p.book.table[0, 0] = int(p.book.free[-1])
    p.free([0, 1])


def test_a_damaged_free_list_is_counted():
    """A count past the list is cut to it, an id that is none is not handed out."""
    pool = api.BlockPool.new(6, 16, 4, 2, 4)
    pool.free_count.fill_(100)
    pool.free_list[5] = 999                      # the first to be taken
    pool.extend(_i32([0]), _i32([8]))
    assert pool.table[0].tolist() == [-1, 1, -1, -1] and int(pool.err_count) == 1 and int(pool.free_count) == 4
    pool.free_count.fill_(-3)
    pool.extend(_i32([1]), _i32([4]))
    assert pool.table[1].tolist() == [-1] * 4 and int(pool.err_count) == 2 and int(pool.free_count) == 0
    assert pool.ref_count.tolist() == [0, 1, 0, 0, 0, 0]


def test_many_blocks_and_rows():
    """More ids than one workgroup ranks, rows longer than one workgroup's pass, blocks of several parts."""
    bt, width, rows = 16, 1100, 6
    p = Pair(3000, 40000, bt, rows, width)
    p.extend([0, 1, 2], [bt * 1100, bt * 901 + 3, 17])
    p.fork([0, 1], [3, 4], [bt * 1050 + 5, bt * 901 + 3])
    p.free([0])
    p.compact()
    p.extend([5], [bt * 600])
    p.free([1, 3])
    p.compact()


def test_a_pool_of_many_small_blocks():
    """More ids than a workgroup counts by itself."""
    width, rows = 1100, 20
    p = Pair(33000, 16, 1, rows, width)
    p.extend(list(range(rows)), [width - 7 * i for i in range(rows)])
    p.free([2, 19, 7, 7])
    p.extend([7], [width])
    p.free([r for r in range(rows) if r not in (0, 5, 7)])
    p.compact()
    p.fork([0, 5], [1, 2], [1000, 40])
    p.free([0])
    p.compact()


def test_blocks_past_32_bit_offsets():
    pool = api.BlockPool.new(4200, 1 << 20, 16, 2, 2)
    pool.cache[4199] = 7
    pool.copy(_i32([4199]), _i32([4150]))
    torch.cuda.synchronize()
    assert bool((pool.cache[4150] == 7).all()) and not bool(pool.cache[4149].any()) and not bool(pool.cache[4151].any())


def test_captured_calls():
    """extend, fork and free in a graph, replayed with eager work between."""
    pool = api.BlockPool.new(64, 256, 16, 4, 8)
    twin = api.BlockPool.new(64, 256, 16, 4, 8)
    args = _i32([0]), _i32([100]), _i32([1]), _i32([2])

    def step(p):
        p.extend(args[0], args[1])
        p.fork(args[0], args[2], args[1])
        p.free(args[0])
        p.fork(args[2], args[0], args[1])
        p.free(args[2])

    step(twin)
    step(pool)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(pool)
    for _ in range(3):
        graph.replay()
        step(twin)
        torch.cuda.synchronize()
        for a, b in ((pool.table, twin.table), (pool.ref_count, twin.ref_count), (pool.free_list, twin.free_list),
                     (pool.free_count, twin.free_count), (pool.cache, twin.cache)):
            assert torch.equal(a, b)
