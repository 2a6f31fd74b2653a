"""The example service's forks and beams without a GPU: what they keep, and alternatives that are none."""
import math

import pytest
import torch

from paper_2311_10359_amd import binding, service

SIZES = service.Sizes(layers=1, q_heads=2, kv_heads=1, dim=64, block=16, blocks=40, vocabulary=16)


class Calls:
    """Stands for the calls, which are left out: lengths and forks by the definition, no blocks; alternatives as given, one list for each score."""

    def __init__(self, *tops):
        self.tops, self.longest, self.parents, self.inputs = list(tops), [], [], []

    def __call__(self, name, sizes, f, *args, **more):
        if name == "plan":
            cached, added = args[:2]
            return binding.CachePlan(cached + added, None, None, None, torch.tensor([0, 0], dtype=torch.int32))
        if name == "fork":
            table, lengths, parents = args[:3]
            self.parents.append(parents.tolist())
            new = torch.where(parents < 0, 0, lengths[parents.clamp(min=0).long()]).int()
            return binding.CacheFork(torch.full((len(parents), table.shape[1]), -1, dtype=torch.int32), new, None, args[5].clone(),
                                     torch.tensor([0, 0, args[5].numel()], dtype=torch.int32))
        if name == "score":
            tokens, logprob = self.tops.pop(0)
            return binding.TokenScores(None, None, None, torch.tensor(tokens, dtype=torch.int32), torch.tensor(logprob))
        if name == "cache attention":
            self.longest.append(more["max_length"])
            return binding.Attention(torch.zeros_like(args[0]), None)
        if name == "prompt attention":
            return binding.Attention(torch.zeros_like(args[0]), None)
        if name == "to queries, keys, values":
            self.inputs.append(args[0].clone())
        return None if name in ("append", "copy") else f(*args, **more)


def tokens(n):
    return torch.zeros((n, SIZES.hidden), dtype=torch.bfloat16)


def parents(*of):
    return torch.tensor(of, dtype=torch.int32)


def begun(lengths=(40, 5), longest=64):
    s, calls = service.Service(SIZES, len(lengths), longest, device="cpu"), Calls()
    s.prompts(calls, tokens(sum(lengths)), list(lengths))
    return s, calls


def test_the_longest_request_is_one_that_is_left():
    """The attention is told no length beyond the table, which the requests that are left fit into."""
    s, calls = begun((60, 5))
    s.fork(calls, parents(1, 1))
    for _ in range(20):
        s.step(calls, tokens(2))
    assert calls.longest == list(range(6, 26)) and s.lengths.tolist() == [25, 25]


def test_a_fork_to_nothing_leaves_no_tokens():
    """... and prompts can come again, of requests that have none in the cache."""
    s, calls = begun()
    s.fork(calls, parents(-1, -1, -1))
    assert s.longest == 0
    s.prompts(calls, tokens(9), [2, 3, 4])
    assert s.lengths.tolist() == [2, 3, 4]
    s.fork(calls, parents())
    assert s.longest == 0 and s.lengths.numel() == 0
