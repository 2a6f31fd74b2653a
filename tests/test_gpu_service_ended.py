"""Requests that end: the example service goes on with those that are left, and with new ones where none is."""
import pytest
import torch

from paper_2311_10359_amd import service

pytestmark = pytest.mark.gpu
SIZES = service.Sizes(layers=2, q_heads=4, kv_heads=2, dim=64, block=16, blocks=40, vocabulary=64, rotary=32)


def run(name, _, f, *args, **more):
    return f(*args, **more)


def tokens(n, seed):
    return torch.randn((n, SIZES.hidden), generator=torch.Generator(device="cuda:0").manual_seed(seed), device="cuda:0").to(torch.bfloat16)


def test_steps_after_the_longest_request_has_ended():
    """Two requests of 60 and 5 tokens in a table of 64; the short one goes on alone, to more tokens than the long one had left."""
    x, got = tokens(65, 2), []
    for longest in (64, 512):
        s = service.Service(SIZES, 2, longest, seed=1)
        s.prompts(run, x, [60, 5])
        s.fork(run, torch.tensor([1], dtype=torch.int32, device="cuda:0"))
        got.append([s.step(run, tokens(1, 3 + i)) for i in range(59)])
        assert s.lengths.tolist() == [64] and s.longest == 64
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_prompts_where_every_request_has_ended():
    s = service.Service(SIZES, 2, 64, seed=1)
    s.prompts(run, tokens(65, 2), [60, 5])
    s.fork(run, torch.tensor([-1, -1, -1], dtype=torch.int32, device="cuda:0"))
    assert s.free.numel() == SIZES.blocks
    fresh = service.Service(SIZES, 3, 64, seed=1)
    x = tokens(30, 4)
    assert torch.equal(s.prompts(run, x, [9, 1, 20]), fresh.prompts(run, x, [9, 1, 20]))
    y = tokens(3, 5)
    assert torch.equal(s.step(run, y), fresh.step(run, y)) and s.lengths.tolist() == [10, 2, 21]
