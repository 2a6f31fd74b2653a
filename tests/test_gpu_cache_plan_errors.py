"""Plans that fail while many workgroups are at work: each of them fails, whichever sees the others' word first.

A call that succeeds goes before, so that the right sums are what a workgroup's shared memory still holds."""
import numpy as np
import pytest
import torch

from paper_2311_10359_amd import binding
from test_gpu_cache_plan import i32

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BLOCK = 16


class Guarded:
    """Outputs and the table in the middle of memory that nothing may write."""

    def __init__(self, n, width, tokens):
        room = binding.fikit_cache_pieces(tokens, n, BLOCK)
        self.whole = {}
        self.table = self._inside("table", n * width).reshape(n, width)
        self.out = binding.CachePlan(self._inside("lengths", n), self._inside("offsets", n + 1), self._inside("slots", tokens, torch.int64),
                                     self._inside("pieces", 4 * room).reshape(room, 4), self._inside("counts", 2))

    def _inside(self, name, size, dtype=torch.int32, most=4096):
        self.whole[name] = torch.full((size + 2 * most,), 9, dtype=dtype, device=DEV)
        return self.whole[name][most:most + size]

    def untouched(self, names):
        return all(bool((self.whole[name] == 9).all()) for name in names)

    def guards_untouched(self):
        return all(bool((x[:4096] == 9).all()) and bool((x[-4096:] == 9).all()) for x in self.whole.values())


# up to 1024 requests and up to 4096 in one launch, two beyond; tokens for more workgroups than run at once
@pytest.mark.parametrize("n, each", [(200, 2000), (3000, 140), (20000, 20)])
@pytest.mark.parametrize("wrong", ["long", "negative", "full"])
def test_nothing_is_written_after_an_error(n, each, wrong):
    tokens = n * each
    width = -(-each // BLOCK)
    rng = np.random.default_rng(n)
    good_cached, good_added = i32([0] * n), i32([each] * n)
    free = torch.arange(n * width, dtype=torch.int32, device=DEV)
    bad_cached, bad_added = good_cached.clone(), good_added.clone()
    at = [int(r) for r in rng.integers(0, n, 3)] + [0, n - 1]
    for r in at:
        if wrong == "long":                 # (the sum of new tokens stays what it is)
            bad_cached[r] = width * BLOCK
        elif wrong == "negative":
            bad_cached[r] = -16
    want = binding.FIKIT_CACHE_FULL if wrong == "full" else binding.FIKIT_INVALID_ARG
    words, guarded = [], []
    for _ in range(6):
        g = Guarded(n, width, tokens)
        word, other = i32([0]), Guarded(n, width, tokens)
        binding.fikit_cache_plan(good_cached, good_added, tokens, BLOCK, other.table, free, word, out=other.out)
        binding.fikit_cache_plan(bad_cached, bad_added, tokens, BLOCK, g.table, free[:-1] if wrong == "full" else free, word, out=g.out)
        words.append(word)
        guarded.append((g, other))
    for word, (g, other) in zip(words, guarded):
        assert int(word) == want
        assert g.untouched(g.whole)
        assert other.guards_untouched() and torch.equal(other.table.reshape(-1), free)
