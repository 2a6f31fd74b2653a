"""A fork refuses lists of free blocks that name a block in use, or one twice: it would be handed out while somebody holds it."""
import pytest

from paper_2311_10359_amd import binding
from test_gpu_fork_free_lists import LENGTHS, PARENTS, SIZES, TABLE, fork, int32, many

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_blocks", SIZES)
@pytest.mark.parametrize("held", [4, 3, 1, 7])
def test_a_free_block_that_is_in_use(n_blocks, held):
    """By a request that goes on (its last block or a whole one) or by one that ends, whose blocks are given back by this fork."""
    for count in (1, 2, 3, 20, 28):
        for at in {0, 1, 2, count - 1}:
            if at < count:
                free = many(n_blocks, count)
                free[at] = held
                for parents in (PARENTS, [-1, -1], [0, 1]):
                    status, _, kept = fork(n_blocks, free, parents)
                    assert status == binding.FIKIT_INVALID_ARG and kept, (count, at, parents)


@pytest.mark.parametrize("n_blocks", SIZES)
def test_a_free_block_that_is_listed_twice(n_blocks):
    """Both taken, one of them, none."""
    for count in (2, 3, 5, 20, 28):
        for first in (0, 1, 2, count - 2):
            for second in (1, 2, count - 1):
                if first < second < count:
                    free = many(n_blocks, count)
                    free[second] = free[first]
                    for parents in (PARENTS, [0], []):
                        status, _, kept = fork(n_blocks, free, parents)
                        assert status == binding.FIKIT_INVALID_ARG and kept, (count, first, second, parents)


def test_far_behind():
    """At either end of the cache and of long lists."""
    for n_blocks in (32768, 1 << 20):
        free = many(n_blocks, n_blocks)
        for at, block in ((len(free) - 1, free[0]), (len(free) - 1, free[-2]), (1, free[0]), (len(free) // 2, 7)):
            changed = list(free)
            changed[at] = block
            assert fork(n_blocks, changed)[0] == binding.FIKIT_INVALID_ARG
        assert fork(n_blocks, free)[0] == 0


@pytest.mark.parametrize("n_blocks", SIZES)
def test_which_error_it_is(n_blocks):
    """A list that cannot be comes before blocks that are too few, whichever workgroup finds its own first."""
    for _ in range(10):
        assert fork(n_blocks, [], [0] * 5)[0] == binding.FIKIT_CACHE_FULL       # 4 needed, 3 given back
        assert fork(n_blocks, [9], [0] * 6)[0] == binding.FIKIT_CACHE_FULL
        assert fork(n_blocks, [9, 9], [0] * 9)[0] == binding.FIKIT_INVALID_ARG
        assert fork(n_blocks, [3], [0] * 9)[0] == binding.FIKIT_INVALID_ARG
        assert fork(n_blocks, [-1], [0] * 9)[0] == binding.FIKIT_INVALID_ARG
        assert fork(n_blocks, [9], [0] * 5)[0] == 0


def test_the_tables_rows_alone_say_what_is_in_use():
    """What lies behind a request's blocks is not looked at, so a block there may be free."""
    for n_blocks in SIZES:
        status = int32([0])
        binding.fikit_cache_fork(int32([[3, 4, 9], [1, 2, 7]], 2, 3), int32(LENGTHS), int32(PARENTS), 16, n_blocks, int32([9, 8]), status)
        assert int(status) == 0 and TABLE[0][2] == -1
