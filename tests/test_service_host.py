"""The binding's choice of streams and the example service's bookkeeping, without a GPU."""
from types import SimpleNamespace

import pytest
import torch

from paper_2311_10359_amd import binding, service

SIZES = service.Sizes(layers=1, q_heads=2, kv_heads=1, dim=64, block=16, blocks=8, vocabulary=16)


def test_a_stream_of_another_device_is_refused():
    """The call would run on the tensors' device, on a stream that nobody named."""
    with pytest.raises(ValueError):
        binding._elsewhere(SimpleNamespace(device=torch.device("cuda", 1)), torch.device("cuda", 0))


class Fake:
    """Stands for the calls: a plan of the lengths, zeros for everything else; leaves `status` behind."""

    def __init__(self, status=0):
        self.status, self.names = status, []

    def __call__(self, name, sizes, f, *args, **more):
        self.names.append(name)
        if name == "plan":
            cached, added, n, _, _, _, word = args
            word.fill_(self.status)
            lengths = cached + added if self.status == 0 else torch.full_like(cached, 12345)       # (unspecified after an error)
            return binding.CachePlan(lengths, torch.zeros(len(cached) + 1, dtype=torch.int32), None, None, torch.tensor([3, 3], dtype=torch.int32))
        if name == "append":
            return None
        if "attention" in name:
            return binding.Attention(torch.zeros_like(args[0]), None)
        return f(*args)


def tokens(n):
    return torch.zeros((n, SIZES.hidden), dtype=torch.bfloat16)


def test_prompts_are_not_continued():
    """No call lets several new tokens of a request see those in the cache, so prompts after others would see too little."""
    s = service.Service(SIZES, 2, 64, device="cpu")
    s.prompts(Fake(), tokens(9), [4, 5])
    record = Fake()
    with pytest.raises(ValueError):
        s.prompts(record, tokens(3), [1, 2])
    assert record.names == [] and s.lengths.tolist() == [4, 5] and s.taken == 3
    s.step(Fake(), tokens(2))
    with pytest.raises(ValueError):
        s.prompts(Fake(), tokens(3), [1, 2])
    one_token_first = service.Service(SIZES, 2, 64, device="cpu")
    one_token_first.step(Fake(), tokens(2))
    with pytest.raises(ValueError):
        one_token_first.prompts(Fake(), tokens(3), [1, 2])


def test_a_step_that_fails_leaves_the_service_as_it_was():
    s = service.Service(SIZES, 2, 64, device="cpu")
    s.prompts(Fake(), tokens(9), [4, 5])
    with pytest.raises(binding.FikitError) as e:
        s.step(Fake(binding.FIKIT_CACHE_FULL), tokens(2))
    assert e.value.status == binding.FIKIT_CACHE_FULL
    assert s.lengths.tolist() == [4, 5] and s.taken == 3 and s.longest == 5 and int(s.status) == 0
    s.step(Fake(), tokens(2))
    assert s.lengths.tolist() == [5, 6]


def test_a_fork_that_fails_leaves_the_service_as_it_was():
    s = service.Service(SIZES, 2, 64, device="cpu")
    s.prompts(Fake(), tokens(9), [4, 5])
    table, free = s.table, s.free

    def record(name, sizes, f, *args, **more):
        if name == "fork":
            args[-1].fill_(status)
            return binding.CacheFork(torch.ones((3, 4), dtype=torch.int32), torch.tensor([4, 4, 5], dtype=torch.int32), None, torch.arange(8, dtype=torch.int32),
                                     torch.tensor([1, 0, 5], dtype=torch.int32))
        assert name == "copy" and args[0] is s.caches
    status = binding.FIKIT_CACHE_FULL
    with pytest.raises(binding.FikitError):
        s.fork(record, torch.tensor([0, 0, 1], dtype=torch.int32))
    assert s.table is table and s.free is free and s.taken == 3 and s.lengths.tolist() == [4, 5] and int(s.status) == 0
    status = binding.FIKIT_OK
    s.fork(record, torch.tensor([0, 0, 1], dtype=torch.int32))
    assert s.lengths.tolist() == [4, 4, 5] and s.taken == 0 and s.free.tolist() == [0, 1, 2, 3, 4]
