"""Attention of one query per request over the 8-bit cache, against 64 bits."""
import math

import numpy as np
import pytest
import torch

import serve_model as model
from paper_2311_10359_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


class Case:
    """A cache whose unowned places, and places behind the requests' ends, hold NaN; a table whose unused entries are no blocks."""

    def __init__(self, seed, lengths, q_heads, kv_heads, dim, block, dtype, spread=1.0, extra_blocks=2):
        gen = torch.Generator().manual_seed(seed)
        self.lengths, self.block, self.dtype, self.scale = lengths, block, dtype, 1 / math.sqrt(dim)
        used = [-(-n // block) for n in lengths]
        n_blocks = sum(used) + extra_blocks
        order = torch.randperm(n_blocks, generator=gen)
        shape = (n_blocks, kv_heads, block, dim)
        self.codes = [(torch.randn(shape, generator=gen) * 60).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8) for _ in range(2)]
        self.exps = [torch.randint(119, 123, shape[:2], generator=gen, dtype=torch.uint8) for _ in range(2)]
        self.table = torch.full((len(lengths), max(used + [1]) + 1), -1, dtype=torch.int32)
        at, owned = 0, torch.zeros(n_blocks, block, dtype=torch.bool)
        for r, n in enumerate(lengths):
            self.table[r, :used[r]] = order[at:at + used[r]].int()
            for i in range(used[r]):
                owned[order[at + i], :min(block, n - i * block)] = True
            at += used[r]
        for c in self.codes:
            c.masked_fill_(~owned[:, None, :, None], 0x7f)
        self.q = (torch.randn((len(lengths), q_heads, dim), generator=gen) * spread).to(dtype)

    def run(self, **more):
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        c = [t.to(DEV) for t in (*self.codes, *self.exps)]
        got = binding.fikit_cache_attention(self.q.to(DEV), *c, self.table.to(DEV), torch.tensor(self.lengths, dtype=torch.int32, device=DEV),
                                            self.scale, status, **more)
        binding.fikit_check_status(status)
        return got

    def check(self, got):
        for r, n in enumerate(self.lengths):
            k, v = (model.cache_values(c, e, self.table[r], n, self.block) for c, e in zip(self.codes, self.exps))
            want = model.Rows(self.q[r:r + 1], k, v, self.scale, [n], self.dtype)
            assert model.near(got.out[r:r + 1], want.out, want.bound), (r, n)
            if got.lse is not None:
                assert model.near(got.lse[r:r + 1], want.lse, want.lse_bound), (r, n)


LENGTHS = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 255, 256, 257, 511, 700]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dim, block", [(64, 16), (64, 64), (128, 16), (128, 32), (128, 128), (128, 256)])
def test_lengths(dim, block, dtype):
    c = Case(dim + block, LENGTHS, 8, 2, dim, block, dtype)
    c.check(c.run())


@pytest.mark.parametrize("q_heads, kv_heads", [(1, 1), (5, 5), (6, 2), (16, 1), (17, 1), (33, 1), (48, 3), (64, 2)])
def test_head_layouts(q_heads, kv_heads):
    c = Case(q_heads, [0, 5, 40, 130, 300], q_heads, kv_heads, 64, 32, torch.bfloat16)
    c.check(c.run())
    c = Case(q_heads, [5, 300], q_heads, kv_heads, 128, 16, torch.float16)
    c.check(c.run())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("lengths, block", [([9000], 16), ([5000, 1, 0, 4097], 64), ([20000], 256), ([4096, 8192], 32)])
def test_contexts_of_many_parts(lengths, block, dtype):
    for dim in (64, 128):
        c = Case(len(lengths) + dim, lengths, 4, 1, dim, block, dtype)
        c.check(c.run())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_peaked_and_flat_scores(dtype):
    """Queries that give scores of some hundreds, and ones that weigh all tokens alike."""
    for spread in (60.0, 1e-4):
        c = Case(21, [700, 3000, 17], 8, 2, 128, 32, dtype, spread=spread)
        c.check(c.run())


def test_no_lse_longer_bound_and_strided_queries():
    c = Case(22, [100, 900, 3], 8, 4, 64, 32, torch.bfloat16)
    plain = c.run()
    bare = c.run(want_lse=False)
    assert bare.lse is None and torch.equal(bare.out, plain.out)
    c.check(c.run(max_length=30 * 32))
    wide = torch.zeros(3, 12, 64, dtype=torch.bfloat16)
    wide[:, 2:10] = c.q
    c.q = wide.to(DEV)[:, 2:10]
    assert not c.q.is_contiguous()
    got = c.run()
    assert torch.equal(got.out, plain.out) and torch.equal(got.lse, plain.lse)


def test_twice_the_same_and_on_another_stream():
    c = Case(23, [3000, 1, 12000, 700], 8, 2, 128, 16, torch.bfloat16)
    first = c.run()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    second = c.run(stream=stream)
    stream.synchronize()
    assert torch.equal(first.out, second.out) and torch.equal(first.lse, second.lse)


def test_nan_among_what_is_seen():
    c = Case(24, [200, 90], 4, 2, 64, 16, torch.bfloat16)
    page = c.table[0, 3]
    c.codes[0][page, 0, 5, 7] = 0x7f            # a key of head 0: its two query heads
    c.codes[1][c.table[1, 1], 1, 2, 9] = 0x7f   # one dimension of a value of head 1
    got = c.run()
    assert torch.isnan(got.out[0, :2]).all() and torch.isfinite(got.out[0, 2:]).all()
    assert torch.isfinite(got.out[1, :2]).all() and torch.isnan(got.out[1, 2:, 9]).all() and int(torch.isnan(got.out).sum()) == 2 * 64 + 2


def test_blocks_beyond_32_bits():
    n_blocks, heads, block, dim = 70000, 4, 128, 128
    c = Case(25, [300], 8, heads, dim, block, torch.bfloat16, extra_blocks=0)
    d_codes = [torch.zeros((n_blocks, heads, block, dim), dtype=torch.uint8, device=DEV) for _ in range(2)]
    d_exps = [torch.ones((n_blocks, heads), dtype=torch.uint8, device=DEV) for _ in range(2)]
    n = c.codes[0].shape[0]
    for i in range(2):
        d_codes[i][-n:] = c.codes[i].to(DEV)
        d_exps[i][-n:] = c.exps[i].to(DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    table = torch.where(c.table >= 0, c.table + (n_blocks - n), c.table)
    got = binding.fikit_cache_attention(c.q.to(DEV), *d_codes, *d_exps, table.to(DEV), torch.tensor([300], dtype=torch.int32, device=DEV),
                                        c.scale, status)
    binding.fikit_check_status(status)
    c.check(got)


def test_what_the_device_refuses():
    for change in ("block", "long", "negative"):
        c = Case(26, [100, 90], 4, 2, 64, 16, torch.bfloat16)
        more = {}
        if change == "block":
            c.table[1, 2] = c.codes[0].shape[0]
        elif change == "long":
            more = {"max_length": 99}
        else:
            c.lengths = [100, -1]
        with pytest.raises(binding.FikitError) as e:
            c.run(**more)
        assert e.value.status == binding.FIKIT_INVALID_ARG


def test_replays_of_a_graph():
    c = Case(27, [3000, 0, 130], 8, 2, 64, 32, torch.float16)
    want = c.run()
    d = [t.to(DEV) for t in (c.q, *c.codes, *c.exps, c.table, torch.tensor(c.lengths, dtype=torch.int32))]
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    out = binding.Attention(torch.empty_like(want.out), torch.empty_like(want.lse))
    ws = binding.workspace(binding.fikit_cache_attention_workspace_bytes(3, 8, 2, 64, c.table.shape[1] * 32), DEV)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.fikit_cache_attention(*d, c.scale, status, out=out, workspace_buf=ws)
    for _ in range(3):
        out.out.fill_(7)
        out.lse.fill_(7)
        ws.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.out, want.out) and torch.equal(out.lse, want.lse)
        binding.fikit_check_status(status)


def test_more_requests_than_a_workgroup_looks_at():
    """1024 requests are the most whose lengths every workgroup adds up."""
    for n in (1023, 1024, 1025):
        lengths = [(13 * i) % 40 for i in range(n)]
        lengths[n // 2] = 4500
        c = Case(n, lengths, 2, 1, 64, 16, torch.bfloat16)
        c.check(c.run())


def test_a_status_that_is_set_stops_it():
    c = Case(30, [100, 3000], 4, 2, 64, 16, torch.bfloat16)
    d = [t.to(DEV) for t in (c.q, *c.codes, *c.exps, c.table, torch.tensor(c.lengths, dtype=torch.int32))]
    out = binding.Attention(torch.full_like(d[0], 7), None)
    status = torch.tensor([binding.FIKIT_CACHE_FULL], dtype=torch.int32, device=DEV)
    binding.fikit_cache_attention(*d, c.scale, status, out=out)
    assert (out.out == 7).all() and int(status) == binding.FIKIT_CACHE_FULL
