"""Norm and rotation of query and key heads against 64 bits."""
import pytest
import torch

import around_model as model
from paper_2311_10359_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def frequencies(rotary, base=10000.0):
    return (base ** (-torch.arange(0, rotary, 2, dtype=torch.float64) / rotary)).float().to(DEV) if rotary else None


def status_word():
    return torch.zeros(1, dtype=torch.int32, device=DEV)


def normal(seed, *shape, dtype=torch.bfloat16):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64).to(dtype).to(DEV)


def check(q, k, positions, freq, neighbours=False, q_weight=None, k_weight=None, epsilon=1e-6, out=None):
    status = status_word()
    want = [None if x is None else model.rotate(x, w, epsilon, positions, freq, neighbours) for x, w in ((q, q_weight), (k, k_weight))]
    got = binding.fikit_rotate_heads(q, k, positions, freq, status, q_weight=q_weight, k_weight=k_weight, epsilon=epsilon, neighbours=neighbours, out=out)
    binding.fikit_check_status(status)
    for g, w in zip(got, want):
        assert (g is None) == (w is None)
        if g is not None:
            kept = positions.cpu() >= 0
            assert model.near(g[kept], w[0][kept], w[1][kept])
    return got


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("dim, rotary, q_heads, kv_heads, tokens", [
    (64, 64, 16, 16, 1), (64, 16, 3, 1, 7), (64, 48, 17, 5, 33), (64, 0, 4, 4, 5), (128, 128, 32, 8, 1), (128, 128, 9, 3, 65), (128, 64, 8, 8, 300),
    (128, 112, 1, 1, 19), (128, 16, 5, 2, 3), (256, 256, 8, 4, 11), (256, 32, 3, 1, 2), (256, 240, 4, 2, 130)])
def test_sizes(dim, rotary, q_heads, kv_heads, tokens, neighbours, dtype):
    q, k = normal(1, tokens, q_heads, dim, dtype=dtype), normal(2, tokens, kv_heads, dim, dtype=dtype)
    positions = torch.randint(0, 5000, (tokens,), generator=torch.Generator().manual_seed(3), dtype=torch.int32).to(DEV)
    w = [(1 + 0.3 * normal(4 + i, dim, dtype=torch.float32)).to(dtype) for i in range(2)]
    check(q, k, positions, frequencies(rotary), neighbours)
    check(q, k, positions, frequencies(rotary), neighbours, *w)
    check(q, k, positions, frequencies(rotary), neighbours, None, w[1])


@pytest.mark.parametrize("neighbours", [False, True])
def test_in_the_product_and_in_place(neighbours):
    dim, hq, hkv, tokens = 128, 12, 4, 77
    qkv = normal(5, tokens, hq + 2 * hkv, dim)
    before = qkv.clone()
    q, k = qkv[:, :hq], qkv[:, hq:hq + hkv]
    positions = torch.arange(tokens, dtype=torch.int32, device=DEV) + 1000
    w = (1 + 0.3 * normal(6, dim, dtype=torch.float32)).to(torch.bfloat16)
    apart = check(q, k, positions, frequencies(64), neighbours, w, w)
    assert torch.equal(qkv, before) and apart.q.is_contiguous() and apart.k.is_contiguous()
    got = check(q, k, positions, frequencies(64), neighbours, w, w, out=binding.RotatedHeads(q, k))
    assert got.q.data_ptr() == q.data_ptr()
    assert torch.equal(q, apart.q) and torch.equal(k, apart.k) and torch.equal(qkv[:, hq + hkv:], before[:, hq + hkv:])


def test_in_place_head_by_head_and_into_other_heads_of_the_product():
    dim, heads, tokens = 64, 6, 41
    qkv = normal(27, tokens, heads, 3, dim)
    before = qkv.clone()
    q, k = qkv[:, :, 0], qkv[:, :, 1]
    positions = torch.arange(tokens, dtype=torch.int32, device=DEV)
    apart = check(q, k, positions, frequencies(64), True)
    check(q, k, positions, frequencies(64), True, out=binding.RotatedHeads(q, k))
    assert torch.equal(q, apart.q) and torch.equal(k, apart.k) and torch.equal(qkv[:, :, 2], before[:, :, 2])
    qkv.copy_(before)
    check(q, None, positions, frequencies(64), True, out=binding.RotatedHeads(qkv[:, :, 2], None))
    assert torch.equal(qkv[:, :, 2], apart.q) and torch.equal(qkv[:, :, :2], before[:, :, :2])
    for one in (qkv[:1], before[:1]):
        check(one[:, :, 0], one[:, :, 1], positions[:1], frequencies(64), out=binding.RotatedHeads(one[:, :, 0], one[:, :, 1]))
    wide = normal(28, tokens, 9, dim)
    check(wide[:, :4], wide[:, 4:6], positions, frequencies(64), out=binding.RotatedHeads(wide[:, :4], wide[:, 6:8]))


def test_one_side_other_orders_and_shared_inputs():
    positions = torch.arange(9, dtype=torch.int32, device=DEV)
    f = frequencies(64)
    q = normal(7, 9, 5, 64)
    check(q, None, positions, f)
    check(None, q, positions, f, k_weight=normal(8, 64))
    heads_first = normal(9, 5, 9, 64).transpose(0, 1)
    out = torch.zeros((5, 9, 64), dtype=torch.bfloat16, device=DEV).transpose(0, 1)
    check(heads_first, q, positions, f, out=binding.RotatedHeads(out, torch.zeros_like(q)))
    check(q[:, :1].expand(-1, 4, -1), q[:1].expand(9, -1, -1), positions, f)
    gaps = torch.full((9, 5, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    check(q, None, positions, f, out=binding.RotatedHeads(gaps[:, :, 64:], None))
    assert bool((gaps[:, :, :64] == 7).all())


def test_tokens_that_are_left_out():
    tokens = 50
    q, k = normal(10, tokens, 8, 128), normal(11, tokens, 2, 128)
    positions = torch.arange(tokens, dtype=torch.int32, device=DEV)
    positions[torch.tensor([0, 7, 8, 30, 49])] = torch.tensor([-1, -5, -(1 << 31), -2, -1], dtype=torch.int32, device=DEV)
    q[7], k[49] = float("nan"), float("inf")
    out = binding.RotatedHeads(torch.full_like(q, 3.0), torch.full_like(k, 4.0))
    check(q, k, positions, frequencies(128), q_weight=normal(12, 128), out=out)
    assert bool((out.q[positions < 0] == 3).all()) and bool((out.k[positions < 0] == 4).all())
    q0, k0 = q.clone(), k.clone()
    check(q, k, positions, frequencies(128), out=binding.RotatedHeads(q, k))
    assert torch.equal(q[positions < 0].view(torch.int16), q0[positions < 0].view(torch.int16))
    assert torch.equal(k[positions < 0].view(torch.int16), k0[positions < 0].view(torch.int16))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_far_positions(dtype):
    positions = torch.tensor([0, 1, (1 << 17) - 1, (1 << 24) + 1, (1 << 30) + 12345, (1 << 31) - 1], dtype=torch.int32, device=DEV)
    for f in (frequencies(128), frequencies(128, 1e6), torch.linspace(0.1, 3.2, 64, device=DEV), torch.full((64,), 3.1415927, device=DEV)):
        check(normal(13, 6, 4, 128, dtype=dtype), normal(14, 6, 2, 128, dtype=dtype), positions, f)


def test_quarter_turns():
    """Angles on and next to the borders of the quarters, of both signs."""
    turn = torch.tensor([0.0, 0.125, 0.25, 0.375, 0.5, 0.625, 0.75, 0.875, 1.0, -0.125, -0.25, -0.5, -0.75, 100.25, 0.12499999, 0.1250001], dtype=torch.float64)
    f = (turn * 2 * torch.pi).float().to(DEV).repeat(2)
    check(normal(15, 3, 3, 64, dtype=torch.float16), None, torch.tensor([1, 2, 3], dtype=torch.int32, device=DEV), f)


def test_ends_of_the_range():
    """Squares beyond and below 32 bits, zeros, epsilon's ends."""
    x = normal(16, 8, 3, 128).float()
    scale = torch.tensor([1e38, 2.0 ** 64, 1e19, 3e-20, 1e-30, 1e-38, 0.0, 1.0], device=DEV)[:, None, None]
    q = (x.clamp(-3, 3) * scale).to(torch.bfloat16)
    positions = torch.arange(8, dtype=torch.int32, device=DEV)
    w = torch.ones(128, dtype=torch.bfloat16, device=DEV)
    for e in (1e-6, 2.0 ** -126, 1e30, 3.4e38):
        check(q, None, positions, frequencies(128), q_weight=w, epsilon=e)
    check(q, q, positions, None, q_weight=w)
    h = (x.clamp(-3, 3) * torch.tensor([2e4, 100.0, 1e-3, 1e-5, 6e-8, 0.0, 1.0, 2.0], device=DEV)[:, None, None]).to(torch.float16)
    check(h, h, positions, frequencies(64), True, q_weight=torch.ones(128, dtype=torch.float16, device=DEV))


def test_what_is_not_finite_stays_in_its_head():
    for dtype in (torch.bfloat16, torch.float16):
        q = normal(17, 4, 8, 64, dtype=dtype)
        clean = q.clone()
        q[1, 2, 5], q[2, 7, 63], q[3, 0, 0] = float("nan"), float("inf"), float("-inf")
        positions = torch.tensor([3, 4, 5, 0], dtype=torch.int32, device=DEV)
        w = normal(18, 64, dtype=dtype)
        for weight in (w, None):
            a = binding.fikit_rotate_heads(q, None, positions, frequencies(32), status_word(), q_weight=weight).q
            b = binding.fikit_rotate_heads(clean, None, positions, frequencies(32), status_word(), q_weight=weight).q
            odd = torch.zeros((4, 8), dtype=torch.bool, device=DEV)
            odd[1, 2] = odd[2, 7] = odd[3, 0] = True
            assert torch.equal(a[~odd], b[~odd]) and bool((~torch.isfinite(a[odd])).any(-1).all())
        assert torch.equal(a[2, 7, 32:63], clean[2, 7, 32:63])     # (not normed and not turned)


def test_more_tokens_than_workgroups():
    tokens = 300_001
    k = normal(19, tokens, 1, 64)
    positions = (torch.arange(tokens, dtype=torch.int32, device=DEV) * 7) % 1001 - 1
    check(None, k, positions, frequencies(64), k_weight=normal(20, 64))


def test_nothing_and_a_status_that_stops():
    f = frequencies(64)
    none = torch.zeros(0, dtype=torch.int32, device=DEV)
    got = binding.fikit_rotate_heads(normal(1, 0, 4, 64), normal(1, 0, 2, 64), none, f, status_word())
    assert got.q.shape == (0, 4, 64) and got.k.shape == (0, 2, 64)
    q = normal(21, 5, 4, 64)
    before, status = q.clone(), torch.full((1,), -9, dtype=torch.int32, device=DEV)
    binding.fikit_rotate_heads(q, None, torch.ones(5, dtype=torch.int32, device=DEV), f, status, out=binding.RotatedHeads(q, None))
    assert torch.equal(q, before) and int(status) == -9


def test_replayed_and_on_another_stream():
    q, k, f, status = normal(22, 13, 8, 128), normal(23, 13, 2, 128), frequencies(128), status_word()
    positions = torch.arange(13, dtype=torch.int32, device=DEV)
    w = normal(24, 128)
    out = binding.RotatedHeads(torch.zeros_like(q), torch.zeros_like(k))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    binding.fikit_rotate_heads(q, k, positions, f, status, q_weight=w, out=out, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    want = binding.fikit_rotate_heads(q, k, positions, f, status, q_weight=w)
    assert torch.equal(out.q, want.q) and torch.equal(out.k, want.k)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.fikit_rotate_heads(q, k, positions, f, status, q_weight=w, out=out)
    for i in range(4):
        positions += 100 * i
        positions[i] = -1
        q.copy_(normal(30 + i, 13, 8, 128))
        out.q.zero_()
        graph.replay()
        want = binding.fikit_rotate_heads(q, k, positions, f, status, q_weight=w)
        kept = positions >= 0
        assert torch.equal(out.q[kept], want.q[kept]) and not bool(out.q[~kept].any())
    assert int(status) == 0


@pytest.mark.parametrize("neighbours, dtype, dim", [(False, torch.bfloat16, 128), (True, torch.float16, 64), (False, torch.float16, 256)])
def test_large_inputs(neighbours, dtype, dim):
    """From 128 MB on the caches are passed by; every 31st token is compared."""
    tokens, hq, hkv = (1 << 27) // (2 * 40 * dim) + 77, 32, 8
    gen = torch.Generator(device=DEV).manual_seed(25)
    qkv = torch.randn((tokens, hq + 2 * hkv, dim), generator=gen, device=DEV, dtype=torch.float32).to(dtype)
    q, k = qkv[:, :hq], qkv[:, hq:hq + hkv]
    positions = torch.arange(tokens, dtype=torch.int32, device=DEV) % 4001 - 1
    w = normal(26, dim, dtype=dtype)
    some = slice(None, None, 31)
    want = [model.rotate(x[some], w, 1e-6, positions[some], frequencies(dim // 2), neighbours) for x in (q, k)]
    kept = positions[some].cpu() >= 0
    status = status_word()
    apart = binding.fikit_rotate_heads(q, k, positions, frequencies(dim // 2), status, q_weight=w, k_weight=w, neighbours=neighbours)
    binding.fikit_rotate_heads(q, k, positions, frequencies(dim // 2), status, q_weight=w, k_weight=w, neighbours=neighbours, out=binding.RotatedHeads(q, k))
    binding.fikit_check_status(status)
    for got in (apart, (q, k)):
        for g, (y, bound) in zip(got, want):
            assert model.near(g[some][kept.to(DEV)], y[kept], bound[kept])
    assert torch.equal(apart.q[positions >= 0], q[positions >= 0]) and torch.equal(apart.k[positions >= 0], k[positions >= 0])
