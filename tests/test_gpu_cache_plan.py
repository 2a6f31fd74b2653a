"""Plans of a step over the paged cache against the definitions."""
import numpy as np
import pytest
import torch

import serve_model as model
from paper_2311_10359_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def case(seed, n, cached_most, added, block, width_more=0):
    rng = np.random.default_rng(seed)
    cached = rng.integers(0, cached_most + 1, n).tolist()
    added = [int(added(rng)) for _ in range(n)]
    width = max([-(-(c + a) // block) for c, a in zip(cached, added)] + [1]) + width_more
    table = np.full((n, width), -7, np.int32)
    held = [-(-c // block) for c in cached]
    need = sum(-(-(c + a) // block) - h for c, a, h in zip(cached, added, held))
    blocks = rng.permutation(sum(held) + need + 3).astype(np.int32)
    at = 0
    for r, h in enumerate(held):
        table[r, :h] = blocks[at:at + h]
        at += h
    return cached, added, table, blocks[at:]


def check(cached, added, table, free, block, **more):
    n, total = len(cached), sum(added)
    d_table, status = i32(table.tolist()).reshape(table.shape), i32([0])
    got = binding.fikit_cache_plan(i32(cached), i32(added), total, block, d_table, i32(free.tolist()), status, **more)
    binding.fikit_check_status(status)
    want_table = table.copy()
    want = model.plan(cached, added, block, want_table, free)
    assert got.lengths.tolist() == want["lengths"]
    assert got.token_offsets.tolist() == want["offsets"]
    if got.slots is not None:
        assert got.slots.tolist() == want["slots"]
    assert got.pieces.tolist() == want["pieces"]
    assert got.counts.tolist() == want["counts"]
    assert np.array_equal(d_table.cpu().numpy(), want_table)


@pytest.mark.parametrize("block", [16, 64, 256])
@pytest.mark.parametrize("n, cached_most, added", [
    (1, 0, lambda r: 1), (1, 40, lambda r: 0), (3, 100, lambda r: 1), (64, 500, lambda r: 1),
    (65, 500, lambda r: r.integers(0, 2)), (7, 0, lambda r: r.integers(1, 700)), (200, 300, lambda r: r.integers(0, 90)),
    (1024, 64, lambda r: 1), (1025, 64, lambda r: r.integers(0, 3)), (3000, 33, lambda r: r.integers(0, 40) * (r.random() < 0.1)),
    (5, 0, lambda r: 6000),
])
def test_against_the_definitions(n, cached_most, added, block):
    check(*case(n + block, n, cached_most, added, block), block)


def test_exact_ends_of_blocks():
    for block in (16, 32):
        cached = [0, block, block - 1, block + 1, 2 * block, 0, 0, block - 1]
        added = [block, block, 1, block - 1, 0, 2 * block, 1, block + 2]
        table = np.arange(8 * 6, dtype=np.int32).reshape(8, 6)
        check(cached, added, table, np.arange(100, 120, dtype=np.int32), block)


def test_no_requests_no_tokens_and_no_slots():
    check([], [], np.zeros((0, 4), np.int32), np.zeros(0, np.int32), 16)
    check([5, 0, 70], [0, 0, 0], np.full((3, 8), 3, np.int32), np.zeros(0, np.int32), 16)
    check(*case(3, 20, 90, lambda r: r.integers(0, 60), 32, width_more=5), 32, want_slots=False)


def test_many_requests_without_tokens_between_others():
    rng = np.random.default_rng(5)
    n = 20000
    added = np.where(rng.random(n) < 0.001, rng.integers(1, 500, n), 0).tolist()
    cached = [0] * n
    need = sum(-(-a // 16) for a in added)
    check(cached, added, np.full((n, 32), -1, np.int32), np.arange(need, dtype=np.int32), 16)


def test_sums_beyond_32_bits():
    """Lengths each of which could be, whose sum is the number of tokens modulo 2^32."""
    for n in (3, 2000, 9000, 20000):
        added = [0] * n
        added[0], added[n // 2], added[n - 1] = 2 ** 31 - 1, 2 ** 31 - 1, 7
        word = i32([0])
        table = torch.full((n, 4), 9, dtype=torch.int32, device=DEV)
        # (rows of the table that are long enough: the width is what the call is told)
        lib = binding.load()
        out = binding.CachePlan(*(torch.zeros(k, dtype=torch.int32, device=DEV) for k in (n, n + 1)), None,
                                torch.zeros((5, 4), dtype=torch.int32, device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV))
        ws = binding.workspace(lib.fikit_cache_plan_workspace_bytes(n), DEV)
        cached, d_added, free = i32([0] * n), i32(added), i32([1] * 50)
        assert lib.fikit_cache_plan(cached.data_ptr(), d_added.data_ptr(), n, 5, 16, table.data_ptr(), 2 ** 27, free.data_ptr(), 50,
                                    out.lengths.data_ptr(), out.token_offsets.data_ptr(), None, out.pieces.data_ptr(), out.counts.data_ptr(),
                                    word.data_ptr(), ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream) == 0
        assert int(word) == binding.FIKIT_INVALID_ARG and (table == 9).all()


@pytest.mark.parametrize("cached, added, total, width, free, status", [
    ([3, 4], [1, 1], 3, 4, 8, binding.FIKIT_INVALID_ARG),          # tokens do not add up
    ([3, -1], [1, 1], 2, 4, 8, binding.FIKIT_INVALID_ARG),
    ([3, 4], [3, -1], 2, 4, 8, binding.FIKIT_INVALID_ARG),
    ([3, 60], [1, 5], 6, 4, 8, binding.FIKIT_INVALID_ARG),         # longer than its row of the table
    ([2 ** 31 - 1, 0], [1, 1], 2, 4, 8, binding.FIKIT_INVALID_ARG),
    ([0, 16], [33, 1], 34, 4, 3, binding.FIKIT_CACHE_FULL),
    ([0], [1], 1, 4, 0, binding.FIKIT_CACHE_FULL),
])
def test_what_the_device_refuses(cached, added, total, width, free, status):
    table = torch.full((len(cached), width), 9, dtype=torch.int32, device=DEV)
    word = i32([0])
    got = binding.fikit_cache_plan(i32(cached), i32(added), total, 16, table, torch.arange(free, dtype=torch.int32, device=DEV), word)
    with pytest.raises(binding.FikitError) as e:
        binding.fikit_check_status(word)
    assert e.value.status == status
    assert (table == 9).all()
    # a call behind it does nothing
    got.lengths.fill_(77)
    binding.fikit_cache_plan(i32([0]), i32([1]), 1, 16, table[:1], i32([1]), word, out=binding.CachePlan(
        got.lengths[:1], got.token_offsets[:2], None, torch.zeros((1, 4), dtype=torch.int32, device=DEV), got.counts))
    assert int(got.lengths[0]) == 77 and int(word) == status and (table == 9).all()


def test_replays_of_a_graph():
    cached, added, table, free = case(11, 300, 200, lambda r: r.integers(0, 9), 32)
    d_cached, d_added, d_free, word = i32(cached), i32(added), i32(free.tolist()), i32([0])
    first = i32(table.tolist())
    d_table = first.clone()
    out = binding.fikit_cache_plan(d_cached, d_added, sum(added), 32, d_table, d_free, word)
    ws = binding.workspace(1 << 14, DEV)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.fikit_cache_plan(d_cached, d_added, sum(added), 32, d_table, d_free, word, out=out, workspace_buf=ws)
    want = model.plan(cached, added, 32, table, free)
    for _ in range(3):
        d_table.copy_(first)
        for t in out:
            t.fill_(-5)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert out.slots.tolist() == want["slots"] and out.pieces.tolist() == want["pieces"] and out.counts.tolist() == want["counts"]
        assert np.array_equal(d_table.cpu().numpy(), table)
        binding.fikit_check_status(word)


@pytest.mark.parametrize("n", [1023, 1025, 4095, 4096, 4097, 8200, 16383, 16384, 16385, 33000])
def test_on_both_sides_of_one_launch(n):
    check(*case(n, n, 50, lambda r: r.integers(0, 4) if r.random() < 0.9 else r.integers(0, 60), 16), 16)
