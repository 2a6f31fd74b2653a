"""Forks and compactions around the sizes from which on they are several launches: the same numbers on both sides, and no workspace below."""
import numpy as np
import pytest

from paper_2311_10359_amd import binding
from test_gpu_cache_blocks import check_compact, check_fork, some_cache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("requests, width, of_fork, of_compaction", [
    (16, 1024, True, True), (16, 1025, False, True), (1, 16384, True, True), (1, 16385, False, True), (1024, 16, True, True), (1023, 17, False, True),
    (16, 2048, False, True), (16, 2049, False, False), (1, 32769, False, False), (1024, 33, False, False), (2, 40000, False, False)])
def test_entries_of_the_table(requests, width, of_fork, of_compaction):
    """Tables that are full, or nearly, of requests that share blocks; children that are few and many."""
    rng = np.random.default_rng(requests + width)
    block = 16
    for groups, longest in ((1, 16 * width), (4, 16 * width // 3), (1, 5)):
        table, lengths, n_blocks, free = some_cache(rng, requests, min(longest, 16 * 24000 // requests), block, groups, spare=1100, width=width)
        for children in (1, 40, 1024):
            assert (binding.fikit_cache_fork_workspace_bytes(requests, children, width, n_blocks) == 0) == of_fork
            check_fork(table, lengths, [int(p) for p in rng.integers(-1, requests, children)], block, n_blocks, free, width)
        assert (binding.fikit_cache_compact_workspace_bytes(requests, width, n_blocks) == 0) == of_compaction
        check_compact(table, lengths, block, n_blocks, free, width)
