"""Causal attention of packed prompts, against 64 bits."""
import math

import pytest
import torch

import serve_model as model
from paper_2311_10359_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def inputs(seed, lengths, q_heads, kv_heads, dim, dtype, spread=1.0):
    gen = torch.Generator().manual_seed(seed)
    whole = torch.randn((sum(lengths), q_heads + 2 * kv_heads, dim), generator=gen)
    whole[:, :q_heads] *= spread
    whole = whole.to(dtype)
    return whole[:, :q_heads], whole[:, q_heads:q_heads + kv_heads], whole[:, q_heads + kv_heads:]


def offsets_of(lengths):
    offsets = [0]
    for n in lengths:
        offsets.append(offsets[-1] + n)
    return offsets


def run(q, k, v, lengths, scale, **more):
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    got = binding.fikit_prompt_attention(q.to(DEV), k.to(DEV), v.to(DEV), torch.tensor(offsets_of(lengths), dtype=torch.int32, device=DEV), scale,
                                         status, **more)
    binding.fikit_check_status(status)
    return got


def check(q, k, v, lengths, scale, got, rows=None):
    at = 0
    for n in lengths:
        take = range(n) if rows is None or n <= rows else sorted({0, 1, n // 2, n - 1, *range(0, n, n // rows)})
        take = torch.tensor(list(take), dtype=torch.long)
        if n:
            want = model.Rows(q[at:at + n][take], k[at:at + n], v[at:at + n], scale, take + 1, q.dtype)
            assert model.near(got.out[at:at + n].cpu()[take], want.out, want.bound), n
            if got.lse is not None:
                assert model.near(got.lse[at:at + n].cpu()[take], want.lse, want.lse_bound), n
        at += n


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dim", [64, 128])
def test_lengths(dim, dtype):
    lengths = [1, 0, 2, 31, 32, 33, 0, 63, 64, 65, 100, 127, 128, 129, 191, 256, 257, 0]
    q, k, v = inputs(dim, lengths, 4, 2, dim, dtype)
    scale = 1 / math.sqrt(dim)
    check(q, k, v, lengths, scale, run(q, k, v, lengths, scale), rows=40)


@pytest.mark.parametrize("q_heads, kv_heads", [(1, 1), (3, 1), (5, 5), (8, 2), (16, 8), (24, 3), (32, 4)])
def test_head_layouts(q_heads, kv_heads):
    for dim, dtype in ((64, torch.float16), (128, torch.bfloat16)):
        lengths = [70, 300]
        q, k, v = inputs(q_heads, lengths, q_heads, kv_heads, dim, dtype)
        check(q, k, v, lengths, 0.1, run(q, k, v, lengths, 0.1), rows=12)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("lengths", [[1000], [2049, 5], [640, 1100, 513]])
def test_long_prompts(lengths, dtype):
    for dim in (64, 128):
        q, k, v = inputs(3, lengths, 2, 1, dim, dtype)
        check(q, k, v, lengths, 0.125, run(q, k, v, lengths, 0.125), rows=50)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_peaked_flat_and_negative_scales(dtype):
    lengths = [400, 77]
    for spread, scale in ((40.0, 0.1), (1e-3, 0.1), (1.0, -0.2), (1.0, 0.0)):
        q, k, v = inputs(5, lengths, 4, 2, 64, dtype, spread)
        check(q, k, v, lengths, scale, run(q, k, v, lengths, scale), rows=40)


def test_many_short_prompts():
    lengths = [(7 * i) % 5 for i in range(3000)]
    q, k, v = inputs(6, lengths, 2, 1, 64, torch.bfloat16)
    check(q, k, v, lengths, 0.125, run(q, k, v, lengths, 0.125))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dim", [64, 128])
def test_what_is_not_finite_is_seen_by_those_behind_it_only(dim, dtype):
    lengths = [90, 150, 300]
    q, k, v = inputs(7, lengths, 2, 1, dim, dtype)
    inf, nan = float("inf"), float("nan")
    for token, d, x in ((89, 3, inf), (90 + 70, 5, nan), (90 + 149, 60, -inf), (240 + 130, 1, inf), (240 + 131, 1, -inf), (240 + 200, 40, -inf),
                        (240 + 299, 2, nan)):
        v[token, 0, d] = x
    k[240 + 250, 0, 4] = nan
    got = run(q, k, v, lengths, 0.125)
    at = 0
    for n in lengths:
        for i in range(n):      # a row at a time: sums over what it sees, nothing else
            want = model.Rows(q[at + i:at + i + 1], k[at:at + i + 1], v[at:at + i + 1], 0.125, [i + 1], dtype)
            assert model.near(got.out[at + i:at + i + 1], want.out, want.bound), (n, i)
        at += n


def test_no_lse_dense_inputs_other_strides_and_streams():
    lengths = [100, 0, 333]
    q, k, v = inputs(8, lengths, 4, 2, 128, torch.bfloat16)
    first = run(q, k, v, lengths, 0.1)
    assert torch.equal(run(q, k, v, lengths, 0.1, want_lse=False).out, first.out)
    assert torch.equal(run(q.contiguous(), k.contiguous(), v.contiguous(), lengths, 0.1).out, first.out)
    moved = [t.transpose(0, 1).contiguous().to(DEV).transpose(0, 1) for t in (q, k, v)]      # heads first
    assert torch.equal(run(*moved, lengths, 0.1).out, first.out)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    other = run(q, k, v, lengths, 0.1, stream=stream)
    stream.synchronize()
    assert torch.equal(other.out, first.out) and torch.equal(other.lse, first.lse)


@pytest.mark.parametrize("offsets", [[0, 50, 40, 100], [1, 50, 100], [0, 50, 99], [0, 50, 101], [0, -1, 100], [0, 2 ** 31 - 1, 100]])
def test_what_the_device_refuses(offsets):
    q, k, v = (t.to(DEV) for t in inputs(9, [100], 2, 1, 64, torch.bfloat16))
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    binding.fikit_prompt_attention(q, k, v, torch.tensor(offsets, dtype=torch.int32, device=DEV), 0.1, status)
    with pytest.raises(binding.FikitError) as e:
        binding.fikit_check_status(status)
    assert e.value.status == binding.FIKIT_INVALID_ARG


def test_no_tokens():
    q, k, v = inputs(10, [0], 2, 1, 64, torch.bfloat16)
    assert run(q, k, v, [0], 0.1).out.shape == (0, 2, 64)


def test_replays_of_a_graph():
    lengths = [100, 0, 333]
    q, k, v = (t.to(DEV) for t in inputs(11, lengths, 4, 2, 64, torch.float16))
    want = run(q, k, v, lengths, 0.1)
    offsets = torch.tensor(offsets_of(lengths), dtype=torch.int32, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    out = binding.Attention(torch.empty_like(want.out), torch.empty_like(want.lse))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.fikit_prompt_attention(q, k, v, offsets, 0.1, status, out=out)
    for _ in range(3):
        out.out.fill_(7)
        out.lse.fill_(7)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.out, want.out) and torch.equal(out.lse, want.lse)
        binding.fikit_check_status(status)


@pytest.mark.parametrize("n", [63, 64, 65, 66])
def test_numbers_of_prompts_on_both_sides_of_the_ordered_ones(n):
    lengths = [(37 * i) % 290 for i in range(n)]
    q, k, v = inputs(12, lengths, 2, 1, 64, torch.bfloat16)
    check(q, k, v, lengths, 0.125, run(q, k, v, lengths, 0.125), rows=9)
    lengths = [0] * (n - 1) + [130]
    q, k, v = inputs(13, lengths, 2, 1, 128, torch.float16)
    check(q, k, v, lengths, 0.125, run(q, k, v, lengths, 0.125), rows=30)


def test_a_status_that_is_set_stops_it():
    q, k, v = (t.to(DEV) for t in inputs(14, [100], 2, 1, 64, torch.bfloat16))
    out = binding.Attention(torch.full((100, 2, 64), 7.0, dtype=torch.bfloat16, device=DEV), None)
    status = torch.tensor([binding.FIKIT_CACHE_FULL], dtype=torch.int32, device=DEV)
    binding.fikit_prompt_attention(q, k, v, torch.tensor([0, 100], dtype=torch.int32, device=DEV), 0.1, status, out=out)
    assert (out.out == 7).all() and int(status) == binding.FIKIT_CACHE_FULL


@pytest.mark.parametrize("lengths", [[129] * 64, [0] * 63 + [1000], [1000] + [1] * 63, list(range(0, 640, 10)), [2000, 3, 1000, 0, 0, 500, 128, 129],
                                     [1] * 65, [300] * 70, [5] * 40 + [1500] + [7] * 40], ids=str)
def test_every_row_is_written_whatever_the_lengths(lengths):
    """Rows are handed out by a search over the prompts' lengths: each of them once, by the rows' place up to 64 prompts."""
    q, k, v = inputs(3, lengths, 2, 1, 64, torch.bfloat16)
    total = sum(lengths)
    out = binding.Attention(torch.full((total, 2, 64), float("nan"), dtype=torch.bfloat16, device=DEV), torch.full((total, 2), float("nan"), device=DEV))
    got = run(q, k, v, lengths, 0.125, out=out)
    assert bool(torch.isfinite(got.out).all()) and bool(torch.isfinite(got.lse).all())
    check(q, k, v, lengths, 0.125, got, rows=6)
