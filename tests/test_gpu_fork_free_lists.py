"""Lists of free blocks that a fork is given: each entry is a block of the cache that nobody holds, and is there once."""
import pytest
import torch

import around_model as model
from paper_2311_10359_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TABLE, LENGTHS, BLOCK = [[3, 4, -1], [1, 2, 7]], [17, 48], 16
PARENTS = [0, 0, 0, -1]                 # block 4 is copied twice; 1, 2 and 7 are given back
SIZES = [33, 40000]                     # in one launch, and in several


def int32(v, *shape):
    return torch.tensor(v, dtype=torch.int32, device=DEV).reshape(shape or (-1,))


def fork(n_blocks, free, parents=PARENTS):
    """(status, outputs, is what lies around them as it was?)"""
    children = len(parents)
    sizes = [(children, 3), (children,), (children, 2), (n_blocks,), (3,)]
    guard = torch.full((2 * n_blocks + 1000,), 77, dtype=torch.int32, device=DEV)
    inside = torch.zeros(guard.numel(), dtype=torch.bool, device=DEV)
    out, at = [], 64
    for shape in sizes:
        size = torch.Size(shape).numel()
        out.append(guard[at:at + size].view(shape))
        inside[at:at + size] = True
        at += size + 128 - size % 64
    status = int32([0])
    binding.fikit_cache_fork(int32(TABLE, 2, 3), int32(LENGTHS), int32(parents), BLOCK, n_blocks, int32(free), status, out=binding.CacheFork(*out))
    return int(status), out, bool((guard[~inside] == 77).all())


def many(n_blocks, count):
    """Free blocks in an order of their own."""
    return [b for b in range(n_blocks - 1, -1, -1) if b not in (1, 2, 3, 4, 7)][:count]


@pytest.mark.parametrize("n_blocks", SIZES)
@pytest.mark.parametrize("of_a_cache", [33, -1, -2, 40000, 1 << 20, 2 ** 31 - 1, -2 ** 31])
def test_entries_that_are_no_blocks(n_blocks, of_a_cache):
    """Also behind those that are taken, which are two here: they would be in the new list, and counted in it."""
    if 0 <= of_a_cache < n_blocks:
        of_a_cache = n_blocks
    for count in (1, 2, 3, 20):
        for at in {0, 1, 2, count // 2, count - 1}:
            if at < count:
                free = many(n_blocks, count)
                free[at] = of_a_cache
                status, _, kept = fork(n_blocks, free)
                assert status == binding.FIKIT_INVALID_ARG and kept, (count, at)


def test_an_entry_that_is_no_block_far_behind():
    for n_blocks, at in ((32768, 30000), (1 << 20, 1 << 19), (1 << 20, (1 << 20) - 6)):
        free = many(n_blocks, n_blocks)
        free[at] = -1
        assert fork(n_blocks, free)[0] == binding.FIKIT_INVALID_ARG


@pytest.mark.parametrize("n_blocks", SIZES)
def test_the_list_of_the_fork_before_is_given_up_to_its_count(n_blocks):
    """Behind its count a new list holds -1 up to the cache's size; those are no blocks."""
    status, (table, lengths, _, free, counts), _ = fork(n_blocks, many(n_blocks, 12))
    assert status == 0 and counts.tolist() == [2, 3, 13]
    for given, want in ((free, binding.FIKIT_INVALID_ARG), (free[:14], binding.FIKIT_INVALID_ARG), (free[:13], 0)):
        word = int32([0])
        parents = int32([1, 1, -1])
        got = binding.fikit_cache_fork(table, lengths, parents, BLOCK, n_blocks, given.contiguous(), word)
        assert int(word) == want
    for name, w in model.fork(table.tolist(), lengths.tolist(), parents.tolist(), BLOCK, n_blocks, free[:13].tolist()).items():
        assert getattr(got, name).tolist() == w


@pytest.mark.parametrize("n_blocks", SIZES)
@pytest.mark.parametrize("outside", [1, 7])
def test_lists_that_are_right(n_blocks, outside):
    """Of no entry, of all blocks that are not in use, of all but some that somebody else keeps."""
    for count in (0, 1, 2, 3, n_blocks - 5, n_blocks - 5 - outside):
        free = many(n_blocks, count)
        for parents in (PARENTS, [-1], [], [1, 1, 0]):
            status, got, kept = fork(n_blocks, free, parents)
            assert status == 0 and kept
            want = model.fork(TABLE, LENGTHS, parents, BLOCK, n_blocks, free)
            for g, w in zip(got, (want[name] for name in binding.CacheFork._fields)):
                assert torch.equal(g.cpu(), torch.tensor(w, dtype=torch.int32).reshape(g.shape))
