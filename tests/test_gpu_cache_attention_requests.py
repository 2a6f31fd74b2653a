"""Attention over the 8-bit cache at the numbers of requests at which the lengths are looked at in another way."""
import pytest
import torch

import serve_model as model
from test_gpu_cache_attention import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [63, 64, 65])
def test_on_both_sides_of_a_wave(n):
    """Up to 64 requests every wave looks at all lengths by itself, beyond that the workgroup does."""
    for dim, dtype in ((64, torch.float16), (128, torch.bfloat16)):
        lengths = [(13 * i) % 140 for i in range(n)]
        lengths[n // 2], lengths[n - 1] = 3000, 1300
        c = Case(n, lengths, 4, 2, dim, 16, dtype)
        c.check(c.run())


@pytest.mark.parametrize("at", [64, 13063, 13064, 13065, 16499])
def test_more_requests_than_a_thread_looks_at_in_one_turn(at):
    """Beyond 16,384 requests a thread adds up more than 64, here 65; the one that holds a place is looked for 64 at a time."""
    n = 16500
    lengths = [(7 * i) % 6 for i in range(n)]
    lengths[at] = 9000               # several workgroups begin in it; request 65 t + 64 is the last of thread t's
    c = Case(at, lengths, 1, 1, 64, 16, torch.bfloat16)
    got = c.run()
    none = torch.tensor(lengths) == 0
    assert bool(torch.isfinite(got.out).all()) and torch.equal(torch.isinf(got.lse[:, 0].cpu()), none)
    for r in sorted({0, 1, 64, 65, n - 1, at - 1, at, min(at + 1, n - 1), *range(3, n, 131)}):
        m = lengths[r]
        k, v = (model.cache_values(codes, e, c.table[r], m, 16) for codes, e in zip(c.codes, c.exps))
        want = model.Rows(c.q[r:r + 1], k, v, c.scale, [m], torch.bfloat16)
        assert model.near(got.out[r:r + 1], want.out, want.bound), r
        assert model.near(got.lse[r:r + 1], want.lse, want.lse_bound), r
