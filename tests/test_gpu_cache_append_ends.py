"""Keys and values put into the 8-bit cache: entries that only look unused, and values that are not finite at the scale's ends."""
import numpy as np
import pytest
import torch

from paper_2311_10359_amd import binding
from test_gpu_cache_append import check

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("piece", [[-1, 0, 0, 1], [-1, 0, 3, 1], [-1, -1, -1, 1], [-1, -1, 0, -1], [-1, 2, -1, -1], [-1, -1, 0, 0]])
def test_an_entry_is_unused_only_if_all_of_it_says_so(piece):
    """A table that holds no block where a request's last one should be makes such pieces: their tokens would be lost."""
    codes = [torch.full((4, 1, 16, 64), 5, dtype=torch.uint8, device=DEV) for _ in range(2)]
    exps = [torch.full((4, 1), 127, dtype=torch.uint8, device=DEV) for _ in range(2)]
    x = torch.ones(4, 1, 64, dtype=torch.bfloat16, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    binding.fikit_cache_append(*codes, *exps, x, x, torch.tensor([[-1] * 4, piece], dtype=torch.int32, device=DEV), status)
    with pytest.raises(binding.FikitError) as e:
        binding.fikit_check_status(status)
    assert e.value.status == binding.FIKIT_INVALID_ARG
    assert all(bool((c == 5).all()) for c in codes) and all(bool((e == 127).all()) for e in exps)


def test_a_plan_over_a_table_without_the_held_block():
    """Through plan and append together: three tokens are in a block that the table does not have."""
    table = torch.full((1, 2), -1, dtype=torch.int32, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    one = torch.ones(1, dtype=torch.int32, device=DEV)
    plan = binding.fikit_cache_plan(3 * one, one, 1, 16, table, one, status)
    codes = [torch.zeros((4, 1, 16, 64), dtype=torch.uint8, device=DEV) for _ in range(2)]
    exps = [torch.ones((4, 1), dtype=torch.uint8, device=DEV) for _ in range(2)]
    x = torch.ones(1, 1, 64, dtype=torch.bfloat16, device=DEV)
    binding.fikit_cache_append(*codes, *exps, x, x, plan.pieces, status)
    with pytest.raises(binding.FikitError):
        binding.fikit_check_status(status)


@pytest.mark.parametrize("exps", [(254, 255), (253, 254), (1, 2), (2, 4)])
@pytest.mark.parametrize("most", [3.3e38, 1e38, 1.0, 2.0 ** -120])
def test_infinities_and_nan_at_the_ends_of_the_scale(exps, most):
    rng = np.random.default_rng(21)
    x = [torch.from_numpy(rng.uniform(-most, most, (24, 2, 64))).to(torch.bfloat16) for _ in range(2)]
    x[0][1, 0, 5] = float("inf")
    x[0][9, 1, 6] = float("nan")
    x[1][2, 1, 0] = float("-inf")
    x[1][20] = float("nan")
    check(*x, [[2, 0, 4, 8], [0, 8, 3, 2], [1, 10, 1, 14]], 16, 22, exps=exps)


@pytest.mark.parametrize("exps", [(254, 255), (1, 2), (120, 130)])
def test_infinities_and_nan_of_float16_at_the_ends(exps):
    rng = np.random.default_rng(23)
    x = [torch.from_numpy(rng.uniform(-65504, 65504, (24, 2, 128))).to(torch.float16) for _ in range(2)]
    x[0][0] = 2.0 ** -24
    x[0][1, 0, 5] = float("inf")
    x[1][2, 1, 0] = float("-inf")
    x[1][20] = float("nan")
    check(*x, [[2, 0, 4, 8], [0, 8, 3, 2], [1, 10, 1, 14]], 16, 24, exps=exps)
