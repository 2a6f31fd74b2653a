"""Token scores within the bounds of their operations one by one, which do not grow with the logits' size."""
import math

import pytest
import torch

from close_scores import CloseScores
from paper_2311_10359_amd import binding
from test_gpu_token_scores import DEV, TYPES, normal, status_word, tokens_for

pytestmark = pytest.mark.gpu


def check(logits, tokens, top, scale=1.0):
    status = status_word()
    got = binding.fikit_token_scores(logits, tokens, status, scale=scale, n_top=top)
    binding.fikit_check_status(status)
    assert CloseScores(logits, tokens, scale, top).differs(got) == []


# rows and lengths on every way to cut them up: a wave, a workgroup of 4, 8 or 16, parts that are joined
CUTS = [(5, 40), (9, 3000), (2100, 3001), (2100, 8001), (3, 20001), (2, 131072), (1, 500_003), (130, 20001), (520, 20001), (1030, 20001)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows, v", CUTS)
def test_offsets(rows, v, dtype):
    """Values around large numbers of both signs, as far as the type tells them apart, at low and high temperatures."""
    for offset, scale in ((0.0, 1.0), (1000.0, 0.7), (-1000.0, 2.0 ** 6), (30000.0, 1.25)):
        step = max(torch.finfo(dtype).eps * abs(offset), 2.0 ** -10)             # (so that a row has more than one or two values)
        x = (normal(v, rows, v) * max(1.0, 4 * step) + offset).to(dtype).to(DEV)
        check(x, tokens_for(rows, rows, v), 9 if v > 100 else 3, scale)


def test_ranges():
    """The types' whole ranges."""
    for dtype, size in ((torch.float32, 1e4), (torch.float32, 1e-6), (torch.bfloat16, 3e4), (torch.bfloat16, 1e-30), (torch.float16, 6e4)):
        x = (normal(7, 5, 3000).clamp(-1, 1) * size).to(dtype).to(DEV)
        for scale in (1.0, 1e-3, 2.0 ** 10):
            check(x, tokens_for(6, 5, 3000), 9, scale)
    x = (normal(8, 5, 3000).clamp(-1, 1) * 3.3e38).to(torch.bfloat16).to(DEV)
    for scale in (2.0 ** -100, 2.0 ** -60, 2.0 ** -4):
        check(x, tokens_for(6, 5, 3000), 9, scale)
    x = (normal(8, 5, 3000) + 1000).to(DEV)
    check(x, tokens_for(6, 5, 3000), 9, 2.0 ** 10)
    check(x - 2000, tokens_for(6, 5, 3000), 9, 2.0 ** 10)


@pytest.mark.parametrize("dtype", TYPES)
def test_ascending_and_descending(dtype):
    """Every batch of a wave brings a larger logit, or none does; around a large number as well."""
    for rows, v in ((2, 40007), (2, 500_003), (140, 20001)):
        up = torch.linspace(-20, 20, v)
        x = torch.stack([up, up.flip(0)] * (rows // 2))
        for offset, scale in ((0.0, 1.0), (2000.0, 1.0), (-500.0, 3.0)):
            check((x + offset).to(dtype).to(DEV), tokens_for(1, rows, v), 5, scale)


@pytest.mark.parametrize("dtype", TYPES)
def test_masks_of_any_kind(dtype):
    """Minus infinity, the type's lowest value and a large one, in rows around zero and far from it."""
    for mask in (-math.inf, torch.finfo(dtype).min, -30000.0):
        for v in (40, 9000, 300_011):
            x = normal(5, 4, v) + torch.tensor([0.0, 500.0, -500.0, 8.0])[:, None]
            x[0, 3:], x[1, ::2], x[2, :-1], x[3, torch.arange(v) % 1999 != 7] = mask, mask, mask, mask
            for scale in (2.0 ** -10, 0.7, 1.0):
                check(x.to(dtype).to(DEV), tokens_for(4, 4, v), 6, scale)
