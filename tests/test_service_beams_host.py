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


def search(width, first, lengths=(4, 5)):
    s, calls = begun(lengths)
    calls.tops.append(first)
    return service.Beams(s, calls, torch.zeros((len(lengths), SIZES.vocabulary)), width), s, calls


@pytest.mark.parametrize("width", [0, -1, 17, 33])
def test_more_beams_than_alternatives_are_refused(width):
    """At most as many as tokens, and as a score lists."""
    s, calls = begun()
    with pytest.raises(ValueError):
        service.Beams(s, calls, torch.zeros((2, SIZES.vocabulary)), width)
    wide = service.Service(SIZES._replace(vocabulary=100), 2, 64, device="cpu")
    with pytest.raises(ValueError):
        service.Beams(wide, calls, torch.zeros((2, 100)), 33)
    assert calls.parents == [] and s.lengths.tolist() == [40, 5]


def test_the_command_refuses_more_beams_than_alternatives(capsys):
    for beams in ("0", "33"):
        with pytest.raises(SystemExit):
            service.main(["--beams", beams])
        assert "--beams" in capsys.readouterr().err


def test_alternatives_that_are_none_have_no_request():
    """A row with less than `width` tokens left: its other beams are empty requests, which nothing continues."""
    none = -math.inf
    beams, s, calls = search(2, ([[7, 3], [9, -1]], [[-0.5, -1.0], [0.0, none]]))
    assert calls.parents == [[0, 0, 1, -1]] and s.lengths.tolist() == [4, 4, 5, 0]
    # the empty request's own alternatives do not count, whatever they are; request 1 has one beam of two alternatives
    calls.tops.append(([[1, 2], [3, 4], [5, 6], [8, 7]], [[-0.1, -9.0], [-9.0, -9.0], [-0.2, -0.3], [-0.1, -0.1]]))
    assert beams.step(calls).tolist() == [0, 0, 2, 2] == calls.parents[-1]
    assert beams.tokens.tolist() == [1, 2, 5, 6] and torch.allclose(beams.logprob, torch.tensor([-0.6, -9.5, -0.2, -0.3]))
    # nothing is left of request 0 but one
    calls.tops.append(([[-1, -1], [2, -1], [5, 6], [8, 7]], [[none, none], [-0.1, none], [-0.2, -0.3], [-0.01, -0.02]]))
    assert beams.step(calls).tolist() == [1, -1, 3, 3] == calls.parents[-1]
    assert beams.tokens.tolist() == [2, -1, 8, 7] and float(beams.logprob[1]) == none and int(s.lengths[1]) == 0


def test_no_token_puts_in_zeros():
    s, _ = begun()
    x = s.tokens(torch.tensor([3, -1, 15], dtype=torch.int32))
    assert not bool(x[1].any()) and torch.equal(x[0], s.w_tokens[:, 3] * 4) and torch.equal(x[2], s.w_tokens[:, 15] * 4)


def test_scores_that_are_not_numbers_are_an_error():
    """They would be sorted in front of those that are, and nothing else tells of them."""
    nan = math.nan
    with pytest.raises(FloatingPointError):
        search(2, ([[7, 3], [-1, -1]], [[-0.5, -1.0], [nan, nan]]))
    beams, s, calls = search(2, ([[7, 3], [9, 2]], [[-0.5, -1.0], [0.0, -1.0]]))
    before, table = (beams.tokens.tolist(), beams.logprob.tolist()), s.table
    calls.tops.append(([[1, 2], [-1, -1], [5, 6], [8, 7]], [[-0.1, -9.0], [nan, nan], [-0.2, -0.3], [-0.1, -0.1]]))
    with pytest.raises(FloatingPointError):
        beams.step(calls)
    assert (beams.tokens.tolist(), beams.logprob.tolist()) == before and s.table is table and len(calls.parents) == 1
