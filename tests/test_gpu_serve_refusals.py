"""Tensors that the attention calls cannot describe to the library are refused before anything is enqueued."""
import pytest
import torch

from paper_2311_10359_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def i32(*shape):
    return torch.zeros(shape, dtype=torch.int32, device=DEV)


def cache(n=3, heads=2, block=16, dim=64):
    codes, exps = torch.zeros((n, heads, block, dim), dtype=torch.uint8, device=DEV), torch.ones((n, heads), dtype=torch.uint8, device=DEV)
    return codes, codes.clone(), exps, exps.clone()


def refused(call, *args, **more):
    with pytest.raises(ValueError):
        call(*args, **more)


def test_plan():
    good = [i32(3), i32(3), 0, 16, i32(3, 4), i32(5), i32(1)]
    binding.fikit_cache_plan(*good)
    for at, bad in ((0, i32(3).long()), (1, i32(2)), (1, i32(6)[::2]), (1, i32(3).cpu()), (2, -1), (4, i32(2, 4)), (4, i32(3, 8)[:, ::2]), (4, i32(12)),
                    (5, i32(5).float()), (6, i32(2)), (6, None)):
        refused(binding.fikit_cache_plan, *good[:at], bad, *good[at + 1:])
    refused(binding.fikit_cache_plan, *good, out=binding.CachePlan(i32(3), i32(3), None, i32(0, 4), i32(2)))
    refused(binding.fikit_cache_plan, *good, workspace_buf=i32(4))
    with pytest.raises(binding.FikitError) as e:
        binding.fikit_cache_plan(*good[:3], 24, *good[4:])
    assert e.value.status == binding.FIKIT_UNSUPPORTED


def test_append():
    x = torch.zeros((4, 2, 64), dtype=torch.bfloat16, device=DEV)
    good = [*cache(), x, x, torch.full((2, 4), -1, dtype=torch.int32, device=DEV), i32(1)]
    binding.fikit_cache_append(*good)
    for at, bad in ((0, cache(dim=128)[0]), (1, cache()[1].float()), (2, i32(3, 2)), (3, cache(n=2)[3]), (4, x.float()), (4, x.half()), (5, x[:3]),
                    (5, x.transpose(1, 2)), (4, x[:, :1]), (6, i32(2, 3)), (6, i32(2, 8)[:, ::2]), (7, i32(2)), (4, x.cpu()), (0, None)):
        refused(binding.fikit_cache_append, *good[:at], bad, *good[at + 1:])
    with pytest.raises(binding.FikitError) as e:      # an odd stride
        wide = torch.zeros((4, 2, 68), dtype=torch.bfloat16, device=DEV)[:, :, :64]
        binding.fikit_cache_append(*good[:4], wide, wide, *good[6:])
    assert e.value.status == binding.FIKIT_INVALID_ARG


def test_cache_attention():
    q = torch.zeros((3, 4, 64), dtype=torch.bfloat16, device=DEV)
    good = [q, *cache(), i32(3, 2), i32(3), 0.1, i32(1)]
    assert binding.fikit_cache_attention(*good).out.shape == q.shape
    for at, bad in ((0, q.float()), (0, q[:2]), (0, q[:, :, :32]), (1, cache(block=32)[0]), (5, i32(2, 2)), (5, i32(3, 4)[:, ::2]), (6, i32(4)), (7, "x"), (8, i32(3))):
        with pytest.raises((ValueError, TypeError)):
            binding.fikit_cache_attention(*good[:at], bad, *good[at + 1:])
    refused(binding.fikit_cache_attention, *good, out=binding.Attention(q[:2], None))
    refused(binding.fikit_cache_attention, *good, out=binding.Attention(q.float(), None))
    refused(binding.fikit_cache_attention, *good, out=binding.Attention(q.clone(), torch.zeros(3, 3, device=DEV)))
    for more, status in (({"max_length": 33}, binding.FIKIT_INVALID_ARG), ({"workspace_buf": torch.zeros(16, dtype=torch.uint8, device=DEV)}, binding.FIKIT_WORKSPACE_TOO_SMALL)):
        with pytest.raises(binding.FikitError) as e:
            binding.fikit_cache_attention(*good, **more)
        assert e.value.status == status


def test_prompt_attention():
    q, k = torch.zeros((5, 4, 64), dtype=torch.float16, device=DEV), torch.zeros((5, 2, 64), dtype=torch.float16, device=DEV)
    good = [q, k, k.clone(), torch.tensor([0, 2, 5], dtype=torch.int32, device=DEV), 0.1, i32(1)]
    assert binding.fikit_prompt_attention(*good).lse.shape == (5, 4)
    for at, bad in ((0, q.float()), (1, k.bfloat16()), (1, k[:4]), (2, k[:, :1]), (0, q.transpose(0, 2)), (3, good[3].long()), (3, i32(0)), (5, i32(0)), (0, q[0])):
        refused(binding.fikit_prompt_attention, *good[:at], bad, *good[at + 1:])
    with pytest.raises(binding.FikitError) as e:
        binding.fikit_prompt_attention(q[:, :3], *good[1:])
    assert e.value.status == binding.FIKIT_INVALID_ARG
