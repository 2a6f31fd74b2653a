"""Forks, compactions and copies of cache blocks: every number and byte has to be the definition's."""
import numpy as np
import pytest
import torch

import around_model as model
from paper_2311_10359_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def int32(v, *shape):
    return torch.tensor(v, dtype=torch.int32, device=DEV).reshape(shape or (-1,))


def status_word(value=0):
    return torch.tensor([value], dtype=torch.int32, device=DEV)


def some_cache(rng, n_requests, longest, block, groups=1, spare=10, outside=3, width=None, junk=True):
    """(table, lengths, n_blocks, free): requests in groups that share whole blocks, blocks scattered, some that nobody knows."""
    lengths = [int(v) for v in rng.integers(0, longest + 1, n_requests)]
    width = width or max(-(-max(lengths) // block), 1)
    table, blocks = [], iter(range(1 << 30))
    for r in range(n_requests):
        pages = -(-lengths[r] // block)
        first = r // groups * groups
        row = table[first][:int(rng.integers(0, min(lengths[r], lengths[first]) // block + 1))] if r > first else []
        row = row + [next(blocks) for _ in range(pages - len(row))]
        table.append(row)
    n = next(blocks)
    n_blocks = n + spare + outside
    order = rng.permutation(n_blocks)
    rows = [[int(order[b]) for b in row] + [int(rng.integers(-5, 1 << 30)) if junk else -1] * (width - len(row)) for row in table]
    return rows, lengths, n_blocks, [int(b) for b in order[n:n + spare]]


def check_fork(table, lengths, parents, block, n_blocks, free, width):
    status = status_word()
    got = binding.fikit_cache_fork(int32(table, len(lengths), width), int32(lengths), int32(parents), block, n_blocks, int32(free), status)
    want = model.fork(table, lengths, parents, block, n_blocks, free)
    if want is None:
        assert int(status) == binding.FIKIT_CACHE_FULL
        return None
    binding.fikit_check_status(status)
    for name, w in want.items():
        g = getattr(got, name).cpu()
        assert torch.equal(g, torch.tensor(w, dtype=torch.int32).reshape(g.shape)), name
    return got


def check_compact(table, lengths, block, n_blocks, free, width):
    status = status_word()
    got = binding.fikit_cache_compact(int32(table, len(lengths), width), int32(lengths), block, n_blocks, int32(free), status)
    binding.fikit_check_status(status)
    for name, w in model.compact(table, lengths, block, n_blocks, free).items():
        g = getattr(got, name).cpu()
        assert torch.equal(g, torch.tensor(w, dtype=torch.int32).reshape(g.shape)), name
    return got


SIZES = [(1, 1, 16, 1), (1, 40, 16, 1), (3, 100, 32, 1), (8, 500, 16, 4), (65, 300, 64, 1), (100, 2000, 256, 5), (1025, 90, 16, 2), (40, 9000, 16, 8),
         (3000, 200, 32, 3), (1024, 60, 16, 4), (200, 9000, 16, 8)]


@pytest.mark.parametrize("requests, longest, block, groups", SIZES)
def test_forks(requests, longest, block, groups):
    rng = np.random.default_rng(requests + longest)
    table, lengths, n_blocks, free = some_cache(rng, requests, longest, block, groups, spare=2 * requests + 3)
    width = len(table[0])
    for parents in ([], list(range(requests)), [-1], [-1] * 5, [requests - 1] * 3, list(range(requests)) * 2,
                    [int(p) for p in rng.integers(-1, requests, max(1, requests // 2))], [int(p) for p in rng.integers(-1, requests, 2 * requests + 1)]):
        check_fork(table, lengths, parents, block, n_blocks, free, width)


@pytest.mark.parametrize("requests, longest, block, groups", SIZES)
def test_compactions(requests, longest, block, groups):
    rng = np.random.default_rng(7 * requests + longest)
    for spare, outside in ((0, 0), (1, 0), (0, 7), (3, 1), (2 * requests + 5, 2), (20000, 40)):
        table, lengths, n_blocks, free = some_cache(rng, requests, longest, block, groups, spare, outside)
        if n_blocks:
            check_compact(table, lengths, block, n_blocks, free, len(table[0]))


def test_blocks_given_back_serve_the_copies():
    """Nothing is free but what requests that end hold."""
    block, width = 16, 4
    table = [[5, 6, 7, -1], [1, 40, 3, 2], [33, 0, -1, -1]]
    lengths = [40, 64, 20]
    check_fork(table, lengths, [0, 0, 0, 2, 2, 0], block, 41, [], width)
    check_fork(table, lengths, [0, 0, 0, 2, 2, 0], block, 41, [9, 8], width)
    check_fork(table, lengths, [0, 0, 0, 0, 0, 2, 2, 0, 0], block, 41, [9, 8], width)
    assert check_fork(table, lengths, [0] * 8, block, 41, [], width) is None             # 7 needed, 6 given back
    assert check_fork(table, lengths, [0] * 8, block, 41, [9], width) is not None
    assert check_fork(table, lengths, [1] * 60, block, 41, [], width) is not None           # (full blocks need none)


def test_borders_of_the_bitmaps():
    """Numbers of blocks around a word, a slice and a thread's share of words; used blocks at both ends."""
    rng = np.random.default_rng(5)
    for n_blocks in (1, 31, 32, 33, 8191, 8192, 8193, 32768, 32769, 70000):
        for n_used in {0, 1, n_blocks // 3, n_blocks - 1, n_blocks}:
            order = [int(b) for b in rng.permutation(n_blocks)]
            for used in (order[:n_used], list(range(n_blocks))[-n_used:] if n_used else [], list(range(n_used))):
                rest = sorted(set(range(n_blocks)) - set(used))
                width = max(1, n_used)
                check_compact([used + [-1] * (width - n_used)], [16 * n_used], 16, n_blocks, rest, width)
                check_fork([used + [-1] * (width - n_used)], [16 * n_used], [-1], 16, n_blocks, rest, width)


def test_most_requests_and_blocks():
    rng = np.random.default_rng(6)
    n, n_blocks, block, width = 16384, 1 << 20, 16, 60
    lengths = rng.integers(0, block * width + 1, n)
    pages = -(-lengths // block)
    order = rng.permutation(n_blocks).astype(np.int32)
    there = np.arange(width)[None, :] < pages[:, None]
    table = np.full((n, width), -7, dtype=np.int32)
    table[there] = order[:pages.sum()]
    free = order[pages.sum():]
    free = free[:len(free) - 5]
    t, l, f, status = torch.from_numpy(table).to(DEV), int32(lengths.tolist()), torch.from_numpy(free).to(DEV), status_word()
    parents = rng.integers(-1, n, n)
    got = binding.fikit_cache_fork(t, l, int32(parents.tolist()), block, n_blocks, f, status)
    want = model.fork(table.tolist(), lengths.tolist(), parents.tolist(), block, n_blocks, free.tolist())
    for name, w in want.items():
        assert np.array_equal(getattr(got, name).cpu().numpy(), np.array(w)), name
    got = binding.fikit_cache_compact(t, l, block, n_blocks, f, status)
    want = model.compact(table.tolist(), lengths.tolist(), block, n_blocks, free.tolist())
    for name, w in want.items():
        assert np.array_equal(getattr(got, name).cpu().numpy(), np.array(w)), name
    binding.fikit_check_status(status)


@pytest.mark.parametrize("change", [
    dict(parents=[0, 2]), dict(parents=[-2]), dict(parents=[1 << 30]), dict(lengths=[17, -1]), dict(lengths=[17, 65]), dict(lengths=[17, 1 << 31]), dict(table=[[3, 99], [1, 2]]),
    dict(table=[[3, -1], [1, 2]]), dict(table=[[3, 1 << 30], [1, 2]]), dict(free=[99, 5]), dict(free=[-1, 5])])
def test_what_the_device_refuses(change):
    a = dict(table=[[3, 4], [1, 2]], lengths=[17, 32], parents=[0, 0, 0], free=[0, 5])
    a.update(change)
    lengths = torch.tensor(a["lengths"], dtype=torch.int64).to(torch.int32).to(DEV)
    guard = torch.full((400,), 77, dtype=torch.int32, device=DEV)
    children = len(a["parents"])
    out = binding.CacheFork(guard[100:100 + 2 * children].view(children, 2), guard[200:200 + children], guard[220:220 + 2 * children].view(children, 2),
                            guard[300:306], guard[350:353])
    inside = torch.zeros(400, dtype=torch.bool, device=DEV)
    for t in out:
        inside[t.storage_offset():t.storage_offset() + t.numel()] = True
    status = status_word()
    binding.fikit_cache_fork(int32(a["table"], 2, 2), lengths, int32(a["parents"]), 16, 6, int32(a["free"]), status, out=out)
    assert int(status) == binding.FIKIT_INVALID_ARG and bool((guard[~inside] == 77).all())
    if "parents" not in change:
        status = status_word()
        binding.fikit_cache_compact(int32(a["table"], 2, 2), lengths, 16, 6, int32(a["free"]), status)
        assert int(status) == binding.FIKIT_INVALID_ARG


def test_compaction_refuses_a_block_that_is_free_and_in_use_or_free_twice():
    for free in ([4, 5], [5, 5], [0, 5, 0]):
        status = status_word()
        binding.fikit_cache_compact(int32([[3, 4], [1, 2]], 2, 2), int32([17, 32]), 16, 6, int32(free), status)
        assert int(status) == binding.FIKIT_INVALID_ARG


def test_nothing_behind_an_error():
    status = status_word(binding.FIKIT_CACHE_FULL)
    out = binding.fikit_cache_fork(int32([[3, 4]], 1, 2), int32([17]), int32([0, 0]), 16, 6, int32([0, 5]), status)
    full = [torch.full_like(t, 55) for t in out]
    binding.fikit_cache_fork(int32([[3, 4]], 1, 2), int32([17]), int32([0, 0]), 16, 6, int32([0, 5]), status, out=binding.CacheFork(*full))
    assert all(bool((t == 55).all()) for t in full) and int(status) == binding.FIKIT_CACHE_FULL


def caches_of(rng, layers, n_blocks, heads, block, dim):
    def some(*shape):
        return torch.from_numpy(rng.integers(0, 256, shape, dtype=np.uint8)).to(DEV)
    return [(some(n_blocks, heads, block, dim), some(n_blocks, heads, block, dim), some(n_blocks, heads), some(n_blocks, heads)) for _ in range(layers)]


@pytest.mark.parametrize("layers, heads, block, dim, n, rest", [
    (1, 1, 16, 64, 1, 0), (2, 3, 16, 64, 5, 2), (4, 8, 64, 128, 20, 30), (3, 5, 256, 128, 7, 1), (33, 2, 16, 64, 9, 0), (70, 1, 16, 128, 3, 1), (1, 300, 16, 64, 4, 4),
    (2, 2, 32, 64, 6000, 5000)])
def test_copies(layers, heads, block, dim, n, rest):
    rng = np.random.default_rng(layers * n)
    n_blocks = 2 * n + 3
    caches = caches_of(rng, layers, n_blocks, heads, block, dim)
    before = [[t.clone() for t in c] for c in caches]
    order = [int(b) for b in rng.permutation(n_blocks)]
    pairs = list(zip(order[:n], order[n:2 * n]))
    listed = int32([list(p) for p in pairs] + [[-1, -1]] * rest, n + rest, 2)
    if rest > 1:
        listed[-1] = 0                          # (to itself)
    status = status_word()
    binding.fikit_cache_copy(caches, listed, status)
    binding.fikit_check_status(status)
    x, y = (torch.tensor(v, device=DEV) for v in zip(*pairs))
    for c, b in zip(caches, before):
        for t, was in zip(c, b):
            was[y] = was[x]
            assert torch.equal(t, was)


def test_copies_of_nothing_and_refusals():
    rng = np.random.default_rng(8)
    caches = caches_of(rng, 2, 5, 2, 16, 64)
    before = [[t.clone() for t in c] for c in caches]
    status = status_word()
    binding.fikit_cache_copy(caches, int32([], 0, 2), status)
    binding.fikit_cache_copy([], int32([0, 1], 1, 2), status)
    binding.fikit_cache_copy(caches, int32([-1, -1] * 300, 300, 2), status)
    binding.fikit_cache_copy(caches, int32([3, 3, 0, 0], 2, 2), status)
    assert int(status) == 0
    for bad in ([0, 5], [5, 0], [-1, 0], [0, -1], [0, 1 << 30], [-2, 1]):
        status = status_word()
        binding.fikit_cache_copy(caches, int32(bad, 1, 2), status)
        assert int(status) == binding.FIKIT_INVALID_ARG
        binding.fikit_cache_copy(caches, int32([0, 1], 1, 2), status)
    assert all(torch.equal(t, w) for c, b in zip(caches, before) for t, w in zip(c, b))


def test_copies_between_unused_entries():
    rng = np.random.default_rng(18)
    n, n_blocks = 20000, 1000
    for layers, heads, block, dim in ((1, 1, 16, 64), (5, 8, 256, 128)):
        if block == 256:
            n_blocks = 200
        caches = caches_of(rng, layers, n_blocks, heads, block, dim)
        want = [[t.clone() for t in c] for c in caches]
        listed = torch.full((n, 2), -1, dtype=torch.int32)
        order = torch.from_numpy(rng.permutation(n_blocks))
        at = torch.from_numpy(rng.choice(n, n_blocks // 2, replace=False))
        listed[at] = order[:n_blocks // 2 * 2].reshape(-1, 2).int()
        status = status_word()
        binding.fikit_cache_copy(caches, listed.to(DEV), status)
        binding.fikit_check_status(status)
        x, y = order[:n_blocks // 2 * 2].reshape(-1, 2).T.to(DEV)
        for c, b in zip(caches, want):
            for t, was in zip(c, b):
                was[y] = was[x]
                assert torch.equal(t, was)


def test_copies_beyond_32_bits():
    n_blocks, heads, block, dim = 70000, 4, 128, 128
    codes = [torch.zeros((n_blocks, heads, block, dim), dtype=torch.uint8, device=DEV) for _ in range(2)]
    exps = [torch.ones((n_blocks, heads), dtype=torch.uint8, device=DEV) for _ in range(2)]
    codes[0][69999], codes[1][3], exps[0][69999], exps[1][3] = 9, 8, 7, 6
    status = status_word()
    binding.fikit_cache_copy([(*codes, *exps)], int32([[69999, 2], [3, 69998]], 2, 2), status)
    binding.fikit_check_status(status)
    assert bool((codes[0][2] == 9).all()) and bool((codes[1][69998] == 8).all()) and bool((exps[0][2] == 7).all()) and bool((exps[1][69998] == 6).all())
    assert int(codes[0].sum(dtype=torch.int64)) == 2 * 9 * heads * block * dim and int(codes[1].sum(dtype=torch.int64)) == 2 * 8 * heads * block * dim


def test_replayed_and_on_another_stream():
    rng = np.random.default_rng(9)
    table, lengths, n_blocks, free = some_cache(rng, 30, 300, 16, 3, spare=100)
    t, l, f, p, status = int32(table, 30, len(table[0])), int32(lengths), int32(free), int32([int(v) for v in rng.integers(-1, 30, 50)]), status_word()
    first = binding.fikit_cache_fork(t, l, p, 16, n_blocks, f, status)
    second = binding.fikit_cache_compact(t, l, 16, n_blocks, f, status)
    caches = caches_of(rng, 2, n_blocks, 2, 16, 64)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    again = binding.fikit_cache_fork(t, l, p, 16, n_blocks, f, status, stream=side)
    binding.fikit_cache_copy(caches, again.copies, status, stream=side)
    other = binding.fikit_cache_compact(t, l, 16, n_blocks, f, status, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip((*first, *second), (*again, *other)))
    forked, compacted = binding.CacheFork(*(torch.empty_like(x) for x in first)), binding.CacheCompaction(*(torch.empty_like(x) for x in second))
    ws = [torch.empty(max(256, n), dtype=torch.uint8, device=DEV) for n in (binding.fikit_cache_fork_workspace_bytes(30, 50, len(table[0]), n_blocks),
                                                                           binding.fikit_cache_compact_workspace_bytes(30, len(table[0]), n_blocks))]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.fikit_cache_fork(t, l, p, 16, n_blocks, f, status, out=forked, workspace_buf=ws[0])
        binding.fikit_cache_copy(caches, forked.copies, status)
        binding.fikit_cache_compact(t, l, 16, n_blocks, f, status, out=compacted, workspace_buf=ws[1])
    for i in range(4):
        p.copy_(int32([int(v) for v in rng.integers(-1, 30, 50)]))
        was = [[x.clone() for x in c] for c in caches]
        for x in (*forked, *compacted, *ws):
            x.fill_(i)
        graph.replay()
        want = model.fork(table, lengths, p.tolist(), 16, n_blocks, free)
        for name, w in want.items():
            assert getattr(forked, name).tolist() == w
        assert all(torch.equal(a, b) for a, b in zip(second, compacted)) and int(status) == 0
        n = want["counts"][0]
        if n:
            x, y = (torch.tensor(v, device=DEV) for v in zip(*want["copies"][:n]))
            for c, b in zip(caches, was):
                for now, w in zip(c, b):
                    w[y] = w[x]
                    assert torch.equal(now, w)


def test_borders_of_slices():
    """More blocks than one launch takes; where the border falls at ends of lanes' words, of words and of counted slices."""
    rng = np.random.default_rng(12)
    for n_blocks in (40960, 40961):
        order = [int(b) for b in rng.permutation(n_blocks)]
        for n_used in (1, 31, 32, 33, 127, 128, 129, 8191, 8192, 8193, 16384, 24577):
            for used in (order[:n_used], list(range(n_blocks))[-n_used:], list(range(n_used))):
                taken = set(used)
                rest = [b for b in order if b not in taken]
                check_compact([used], [16 * n_used], 16, n_blocks, rest, n_used)
                check_compact([used], [16 * n_used], 16, n_blocks, rest[:n_blocks // 3], n_used)
                check_fork([used], [16 * n_used], [-1], 16, n_blocks, rest, n_used)


@pytest.mark.parametrize("n_blocks", [5, 8192, 40000, 1 << 20])
def test_no_requests(n_blocks):
    rng = np.random.default_rng(13)
    free = [int(b) for b in rng.permutation(n_blocks)]
    for some in (free, free[:n_blocks // 2], []):
        check_fork([], [], [], 16, n_blocks, some, 3)
        status = status_word()
        got = binding.fikit_cache_fork(int32([], 0, 3), int32([]), int32([-1, -1, -1]), 16, n_blocks, int32(some), status)
        binding.fikit_check_status(status)
        assert bool((got.block_table == -1).all()) and bool((got.lengths == 0).all()) and bool((got.copies == -1).all())
        assert got.free_blocks.tolist() == some + [-1] * (n_blocks - len(some)) and got.counts.tolist() == [0, 0, len(some)]
        check_compact([], [], 16, n_blocks, some, 3)


def several_launches(a, children, n_blocks=40000):
    """A fork and a compaction into outputs with a border, from a workspace that holds anything: (statuses, outputs, are the borders as they were?)."""
    t, f = int32(a["table"], 2, 2), int32(a["free"])
    lengths = torch.tensor(a["lengths"], dtype=torch.int64).to(torch.int32).to(DEV)
    sizes = [(2 * children, (children, 2)), (children, (children,)), (2 * children, (children, 2)), (n_blocks, (n_blocks,)), (3, (3,)),
             (4, (2, 2)), (2 * len(f), (len(f), 2)), (len(f), (len(f),)), (2, (2,))]
    guard = torch.full((2 * n_blocks,), 77, dtype=torch.int32, device=DEV)
    inside = torch.zeros(2 * n_blocks, dtype=torch.bool, device=DEV)
    out, at = [], 64
    for size, shape in sizes:
        out.append(guard[at:at + size].view(shape))
        inside[at:at + size] = True
        at += size + 64 - size % 64
    bytes_of = [binding.fikit_cache_fork_workspace_bytes(2, children, 2, n_blocks), binding.fikit_cache_compact_workspace_bytes(2, 2, n_blocks)]
    assert all(bytes_of)
    found = [status_word(a.get("status", 0)) for _ in bytes_of]
    work = [torch.full((n + 64,), 255, dtype=torch.uint8, device=DEV) for n in bytes_of]
    binding.fikit_cache_fork(t, lengths, int32(a["parents"]), 16, n_blocks, f, found[0], out=binding.CacheFork(*out[:5]), workspace_buf=work[0][:bytes_of[0]])
    binding.fikit_cache_compact(t, lengths, 16, n_blocks, f, found[1], out=binding.CacheCompaction(*out[5:]), workspace_buf=work[1][:bytes_of[1]])
    kept = bool((guard[~inside] == 77).all()) and all(bool((w[n:] == 255).all()) for w, n in zip(work, bytes_of))
    return [int(s) for s in found], out, kept


@pytest.mark.parametrize("change", [
    dict(parents=[0, 2]), dict(parents=[-2]), dict(parents=[1 << 30]), dict(lengths=[17, -1]), dict(lengths=[17, 33]), dict(lengths=[17, 1 << 31]),
    dict(table=[[3, 40000], [1, 2]]), dict(table=[[3, -1], [1, 2]]), dict(table=[[3, 1 << 30], [1, 2]]), dict(free=[40000, 5]), dict(free=[-1, 5]),
    dict(free=[6, 5, 6]), dict(free=[1, 5])])
def test_refusals_in_several_launches(change):
    a = dict(table=[[3, 4], [1, 2]], lengths=[17, 32], parents=[0, 0, 0], free=[39999, 5])
    a.update(change)
    statuses, _, kept = several_launches(a, len(a["parents"]))
    assert kept
    if change.get("free") not in ([6, 5, 6], [1, 5]):       # (which a fork does not look at)
        assert statuses[0] == binding.FIKIT_INVALID_ARG
    assert statuses[1] == (0 if "parents" in change else binding.FIKIT_INVALID_ARG)


def test_too_few_and_nothing_behind_an_error_in_several_launches():
    a = dict(table=[[3, 4], [1, 2]], lengths=[17, 31], parents=[0, 0, 0, 1, 1], free=[39999])
    statuses, _, kept = several_launches(a, 5)
    assert kept and statuses == [binding.FIKIT_CACHE_FULL, 0]
    statuses, out, kept = several_launches(dict(a, status=binding.FIKIT_CACHE_FULL), 5)
    assert kept and statuses == [binding.FIKIT_CACHE_FULL] * 2 and all(bool((t == 77).all()) for t in out)


@pytest.mark.parametrize("requests, children", [(4096, 4096), (4096, 4097), (4097, 5), (5, 8192), (8192, 8193), (8193, 300), (16384, 1), (1, 16384)])
def test_how_many_requests_and_children_a_thread_has(requests, children):
    rng = np.random.default_rng(requests + children)
    table, lengths, n_blocks, free = some_cache(rng, requests, 70, 16, groups=3, spare=requests // 2 + children // 3)
    width = len(table[0])
    for parents in (rng.integers(-1, requests, children), np.minimum(rng.geometric(0.01, children) - 1, requests - 1), np.full(children, requests - 1)):
        check_fork(table, lengths, [int(p) for p in parents], 16, n_blocks, free, width)
