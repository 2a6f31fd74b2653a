"""The bounds of token scores tell results that are off from results that are not, whatever the logits' size."""
import math

import pytest
import torch

from close_scores import CloseScores
from paper_2311_10359_amd import binding


def rows(offset):
    return torch.randn((5, 3000), generator=torch.Generator().manual_seed(8)) + offset


def results(scores):
    """As a perfect call leaves them."""
    return binding.TokenScores(*(scores.want[name].float() if name != "top_tokens" else scores.want[name].int() for name in binding.TokenScores._fields))


CASES = [(0, 1.0), (1000, 1.0), (-1000, 1.0), (1000, 2.0 ** 10), (-1000, 2.0 ** 10), (3e4, 0.7)]


@pytest.mark.parametrize("offset, scale", CASES)
def test_what_is_right_is_taken(offset, scale):
    x, tokens = rows(offset), torch.tensor([0, 17, 2999, -1, 1234], dtype=torch.int32)
    scores = CloseScores(x, tokens, scale, 9)
    assert scores.differs(results(scores)) == []


@pytest.mark.parametrize("offset, scale", CASES)
@pytest.mark.parametrize("name", ["logprob", "entropy", "lse", "top_logprob"])
def test_what_is_off_is_refused(offset, scale, name):
    """By a hundredth; log sums of a million and more by a quarter, 4 of whose roundings are that."""
    x, tokens = rows(offset), torch.tensor([0, 17, 2999, 5, 1234], dtype=torch.int32)
    scores = CloseScores(x, tokens, scale, 9)
    got = results(scores)
    large = name == "lse" and abs(offset * scale) > 1e5
    for shift in (0.25, -0.25) if large else (0.01, -0.01):
        values = getattr(got, name)
        for row in range(5):
            changed = values.clone()
            changed[row] += shift
            assert scores.differs(got._replace(**{name: changed})) == [name]


def test_log_probabilities_from_a_rounded_sum_are_refused():
    """z - lse in 32 bits loses what the offset has."""
    for offset, scale in ((1000, 2.0 ** 10), (-1000, 2.0 ** 10), (1000, 1.0)):
        x, tokens = rows(offset), torch.tensor([0, 17, 2999, 5, 1234], dtype=torch.int32)
        scores = CloseScores(x, tokens, scale, 9)
        z = x * scale
        log_p = z - torch.logsumexp(z, 1, keepdim=True)
        got = results(scores)
        top = log_p.gather(1, scores.want["top_tokens"])
        assert scores.differs(got._replace(top_logprob=top)) == ["top_logprob"]
        entropy = -(log_p.exp() * log_p).sum(1)
        assert scores.differs(got._replace(entropy=entropy)) == ["entropy"]
        assert math.isfinite(float(scores.bound["entropy"].max()))


@pytest.mark.parametrize("offset, scale", CASES)
def test_bounds_of_near_tokens_do_not_grow_with_the_offset(offset, scale):
    x, tokens = rows(offset), torch.zeros(5, dtype=torch.int32)
    there, here = CloseScores(x, tokens, scale, 9), CloseScores(x - x.amax(1, keepdim=True), tokens, scale, 9)
    for name in ("entropy", "top_logprob"):
        assert bool((there.bound[name] <= 1.01 * here.bound[name]).all()) and float(there.bound[name].max()) < 0.01
