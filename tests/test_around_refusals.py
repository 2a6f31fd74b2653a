"""What the calls around the attention refuse on the host, before any HIP call; pointers are never followed here."""
import pytest
import torch

from paper_2311_10359_amd import binding

FAKE, ODD, NULL = 0x10000, 0x10001, None
OK, INVALID, SMALL, UNSUPPORTED = 0, binding.FIKIT_INVALID_ARG, binding.FIKIT_WORKSPACE_TOO_SMALL, binding.FIKIT_UNSUPPORTED


def vectors(data=FAKE, token=512, head=64):
    return binding._Vectors(data, token, head)


def rotate(**change):
    a = dict(q=vectors(), k=vectors(0x20000), q_heads=4, kv_heads=2, dim=64, value_type=0, q_weight=FAKE, k_weight=NULL, epsilon=1e-6, positions=FAKE,
             frequencies=FAKE, rotary=64, pairs=0, tokens=5, q_out=vectors(0x30000), k_out=vectors(0x40000), status=FAKE)
    assert set(change) <= set(a)
    a.update(change)
    return binding.load().fikit_rotate_heads(*a.values(), None)


@pytest.mark.parametrize("change, want", [
    (dict(q=vectors(NULL)), INVALID), (dict(q=None), INVALID), (dict(k=vectors(FAKE + 8)), INVALID), (dict(k=vectors(token=4)), INVALID),
    (dict(k_out=vectors(0x40000, head=68)), INVALID), (dict(k_out=None), INVALID), (dict(q_out=vectors(0x30000, head=32)), INVALID),
    (dict(q_out=vectors(0x30000, token=0)), INVALID), (dict(q_out=vectors(0x30000, token=128)), INVALID), (dict(q_out=vectors(0x30000, token=64, head=128)), INVALID),
    (dict(q_out=vectors(0x30000, token=248)), INVALID), (dict(k_out=vectors(0x40000, token=120)), INVALID), (dict(q_out=vectors(0x30000, token=64, head=312)), INVALID), (dict(q_out=vectors(0x30000, head=0)), INVALID),
    (dict(q_out=vectors(FAKE, token=1024)), INVALID), (dict(q_out=vectors(FAKE, head=128)), INVALID),       # in place, of other strides
    (dict(q_out=vectors(0x20000)), INVALID), (dict(k_out=vectors(FAKE)), INVALID), (dict(k_out=vectors(0x30000)), INVALID),
    (dict(q_weight=FAKE + 8), INVALID), (dict(k_weight=ODD), INVALID), (dict(epsilon=0.0), INVALID), (dict(epsilon=-1.0), INVALID),
    (dict(epsilon=float("nan")), INVALID), (dict(epsilon=float("inf")), INVALID), (dict(epsilon=1e-40), INVALID),
    (dict(positions=NULL), INVALID), (dict(positions=ODD), INVALID), (dict(frequencies=NULL), INVALID), (dict(frequencies=ODD), INVALID),
    (dict(status=NULL), INVALID), (dict(status=ODD), INVALID), (dict(tokens=1 << 31), INVALID), (dict(pairs=2), INVALID), (dict(pairs=-1), INVALID),
    (dict(value_type=2), INVALID), (dict(value_type=-1), INVALID), (dict(dim=96), UNSUPPORTED), (dict(dim=512), UNSUPPORTED), (dict(dim=0), UNSUPPORTED),
    (dict(rotary=8), UNSUPPORTED), (dict(rotary=80), UNSUPPORTED), (dict(q_heads=65536), UNSUPPORTED),
    (dict(tokens=0, q=None, positions=NULL), OK), (dict(q_heads=0, kv_heads=0, q=None, k=None), OK),
])
def test_rotate_heads(change, want):
    assert rotate(**change) == want


QUERIES, KEYS = 0x10000, 0x10200        # in one product of 9 heads of 64: queries of 4, keys of 2, values; a token takes 576 values


@pytest.mark.parametrize("q_out, k_out", [
    (vectors(KEYS, 576), vectors(0x30000, 576)), (vectors(QUERIES + 128, 576), vectors(KEYS, 576)), (vectors(0x30000, 576), vectors(KEYS - 128, 576)),
    (vectors(QUERIES + 1152, 576), vectors(0x40000)), (vectors(0x30000), vectors(QUERIES + 128, 640)), (vectors(0x30000), vectors(0x30000 + 128)),
    (vectors(QUERIES, 640), vectors(KEYS, 576)), (vectors(0x30000, 64, 320), vectors(0x30000 + 640, 64, 320))])
def test_rotate_heads_over_each_other(q_out, k_out):
    assert rotate(q=vectors(QUERIES, 576), k=vectors(KEYS, 576), q_out=q_out, k_out=k_out) == INVALID


@pytest.mark.parametrize("q_out, k_out", [(0x10080, 0x10100), (0x10040, 0x30000), (0x30000, 0x30040), (0x10000, 0x10000), (0x10180, 0x30000)])
def test_rotate_heads_over_each_other_head_by_head(q_out, k_out):
    """Query, key and value of 64 each for a head."""
    assert rotate(kv_heads=4, q=vectors(0x10000, 768, 192), k=vectors(0x10080, 768, 192), q_out=vectors(q_out, 768, 192), k_out=vectors(k_out, 768, 192)) == INVALID


def test_rotate_heads_over_each_other_in_one_token():
    assert rotate(tokens=1, q=vectors(QUERIES, 0), k=vectors(KEYS, 0), q_out=vectors(QUERIES + 256, 0), k_out=vectors(0x30000, 0)) == INVALID


def test_rotate_heads_takes_any_epsilon_without_a_norm():
    assert rotate(q_weight=NULL, epsilon=0.0, tokens=0) == OK


def test_rotate_heads_binding():
    x, i = torch.zeros((3, 2, 64), dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    f, status = torch.zeros(32), torch.zeros(1, dtype=torch.int32)
    native = binding._marshal()

    def call(q=x, k=x, positions=i, frequencies=f, q_weight=None, out=None):
        return native.rotate_heads(q, k, positions, frequencies, status, q_weight, None, 1e-6, False, out, 0)
    with pytest.raises(ValueError):
        binding.fikit_rotate_heads(None, None, i, f, status)
    with pytest.raises(ValueError):
        binding.fikit_rotate_heads(x, x, i, f, status)                       # tensors on a GPU
    for bad in (dict(q=x.float()), dict(q=x[0]), dict(k=x[:2]), dict(k=x.half()), dict(k=x[:, :, :32]), dict(positions=i[:2]), dict(positions=i.long()),
                dict(frequencies=f.double()), dict(q_weight=torch.ones(64)), dict(q_weight=torch.ones(32, dtype=torch.bfloat16)), dict(q=None, k=None),
                dict(q=x.clone().requires_grad_()), dict(q_weight=torch.ones(64, dtype=torch.bfloat16, requires_grad=True)), dict(q=None, q_weight=x[0, 0]),
                dict(out=(x,)), dict(out=(x, None)), dict(out=(x[:2], x)), dict(q=x.transpose(1, 2))):
        with pytest.raises(ValueError):
            call(**bad)


def fork(**change):
    a = dict(table=0x1000000, width=3, lengths=0x2000000, n=4, parents=0x3000000, children=5, block=16, n_blocks=100, free=0x4000000, n_free=9, new_table=0x5000000,
             new_lengths=0x6000000, copies=0x7000000, new_free=0x8000000, counts=0x9000000, status=0xa000000, ws=0xb000000, ws_bytes=1 << 20)
    assert set(change) <= set(a)
    a.update(change)
    return binding.load().fikit_cache_fork(*a.values(), None)


def compact(**change):
    a = dict(table=0x1000000, width=3, lengths=0x2000000, n=4, block=16, n_blocks=100, free=0x4000000, n_free=9, new_table=0x5000000, copies=0x7000000,
             new_free=0x8000000, counts=0x9000000, status=0xa000000, ws=0xb000000, ws_bytes=1 << 20)
    assert set(change) <= set(a)
    a.update(change)
    return binding.load().fikit_cache_compact(*a.values(), None)


SHARED = [
    (dict(table=NULL), INVALID), (dict(table=0x1000002), INVALID), (dict(lengths=NULL), INVALID), (dict(lengths=ODD), INVALID), (dict(free=NULL), INVALID),
    (dict(free=ODD), INVALID), (dict(n_free=101), INVALID), (dict(n_blocks=0), INVALID), (dict(new_table=NULL), INVALID), (dict(new_table=ODD), INVALID),
    (dict(copies=NULL), INVALID), (dict(copies=0x7000004), INVALID), (dict(new_free=NULL), INVALID), (dict(new_free=ODD), INVALID), (dict(counts=NULL), INVALID),
    (dict(counts=ODD), INVALID), (dict(status=NULL), INVALID), (dict(status=ODD), INVALID), (dict(n=2000, ws=NULL), INVALID), (dict(n_blocks=40000, ws=0xb000010), INVALID),
    (dict(width=1 << 31), INVALID), (dict(new_table=0x1000000), INVALID), (dict(new_free=0x4000000), INVALID), (dict(new_free=0x4000000 + 32), INVALID),
    (dict(counts=0x2000000), INVALID), (dict(copies=0x5000000), INVALID), (dict(n=2000, ws_bytes=256), SMALL), (dict(n_blocks=40000, ws_bytes=256), SMALL),
    (dict(block=8), UNSUPPORTED), (dict(block=0), UNSUPPORTED),
    (dict(block=48), UNSUPPORTED), (dict(block=512), UNSUPPORTED), (dict(n=16385), UNSUPPORTED), (dict(n_blocks=(1 << 20) + 1), UNSUPPORTED)]


@pytest.mark.parametrize("change, want", SHARED + [(dict(parents=NULL), INVALID), (dict(parents=ODD), INVALID), (dict(new_lengths=NULL), INVALID),
                                                  (dict(new_lengths=ODD), INVALID), (dict(new_lengths=0x3000000), INVALID), (dict(children=16385), UNSUPPORTED)])
def test_fork(change, want):
    assert fork(**change) == want


@pytest.mark.parametrize("change, want", SHARED)
def test_compact(change, want):
    assert compact(**change) == want


def test_block_workspaces():
    for f, sizes in ((binding.fikit_cache_fork_workspace_bytes, (7, 9)), (binding.fikit_cache_compact_workspace_bytes, (7,))):
        assert f(*sizes, 100, 1000) == 0 and 0 < f(*sizes, 100, 40000) <= f(*sizes, 100, 1 << 20) and 0 < f(*sizes, 10000, 1000)
        assert f(*sizes, 100, (1 << 20) + 1) == 0 and f(*(16385 for _ in sizes), 100, 5) == 0 and f(*(2000 for _ in sizes), 1, 5) > 0


def cache(**change):
    a = dict(k=FAKE, v=FAKE, k_exp=FAKE, v_exp=FAKE, n_blocks=10, kv_heads=2, block_tokens=16, head_dim=64)
    assert set(change) <= set(a)
    a.update(change)
    return binding._Cache(*a.values())


def test_copy():
    def call(caches=(cache(),), copies=FAKE, n=3, status=FAKE):
        return binding.load().fikit_cache_copy((binding._Cache * len(caches))(*caches), len(caches), copies, n, status, None)
    for change, want in [(dict(k=NULL), INVALID), (dict(v=ODD), INVALID), (dict(k_exp=NULL), INVALID), (dict(n_blocks=0), INVALID), (dict(kv_heads=0), INVALID),
                         (dict(block_tokens=24), UNSUPPORTED), (dict(head_dim=96), UNSUPPORTED)]:
        assert call((cache(**change),)) == want and call((cache(), cache(**change))) == want
    for change in (dict(n_blocks=11), dict(kv_heads=3), dict(block_tokens=32), dict(head_dim=128)):
        assert call((cache(), cache(**change))) == INVALID
    assert call(copies=NULL) == INVALID and call(copies=FAKE + 4) == INVALID and call(status=NULL) == INVALID and call(n=1 << 31) == INVALID
    assert call(n=0, copies=NULL) == OK and call(()) == OK
    assert binding.load().fikit_cache_copy(None, 1, FAKE, 3, FAKE, None) == INVALID


def test_block_bindings():
    i = torch.zeros(3, dtype=torch.int32)
    table, status, native = torch.zeros((3, 2), dtype=torch.int32), torch.zeros(1, dtype=torch.int32), binding._marshal()
    codes, exps = torch.zeros((4, 2, 16, 64), dtype=torch.uint8), torch.ones((4, 2), dtype=torch.uint8)
    with pytest.raises(ValueError):
        binding.fikit_cache_fork(table, i, i, 16, 9, i, status)              # tensors on a GPU
    for bad in ((table[0], i, i, i), (table, i[:2], i, i), (table, i, i.long(), i), (table, i, i, i.float()), (table.t(), i[:2], i, i)):
        with pytest.raises(ValueError):
            native.cache_fork(bad[0], bad[1], bad[2], 16, 9, bad[3], status, None, None, 0)
    for out in ((i,), (table, i, table, i, i), binding.CacheFork(table, i, table, torch.zeros(9, dtype=torch.int32), i[:2])):
        with pytest.raises(ValueError):
            native.cache_fork(table, i, i, 16, 9, i, status, out, None, 0)
    with pytest.raises(ValueError):
        native.cache_compact(table, i, 16, 9, i, status, binding.CacheCompaction(table, table, i, i), None, 0)
    for caches in ([(codes, codes, exps)], [(codes, codes, exps, exps.long())], [(codes, codes[:2], exps, exps)], [codes]):
        with pytest.raises(ValueError):
            native.cache_copy(caches, table, status, 0)
    with pytest.raises((ValueError, TypeError)):
        native.cache_copy(5, table, status, 0)
    with pytest.raises(ValueError):
        native.cache_copy([(codes, codes, exps, exps)], i, status, 0)


def scores(**change):
    a = dict(logits=0x1000000, value_type=0, stride=70000, rows=4, vocabulary=70000, scale=1.0, tokens=0x10000, n_top=3, logprob=0x20000, entropy=0x30000, lse=0x40000,
             top_tokens=0x50000, top_logprob=0x60000, status=FAKE, ws=FAKE, ws_bytes=1 << 30)
    assert set(change) <= set(a)
    a.update(change)
    return binding.load().fikit_token_scores(*a.values(), None)


@pytest.mark.parametrize("change, want", [
    (dict(logits=NULL), INVALID), (dict(logits=ODD), INVALID), (dict(logits=0x1000002, value_type=2), INVALID),
    (dict(logprob=0x1000000), INVALID), (dict(entropy=0x1000000 + 8 * 70000 - 4), INVALID), (dict(lse=0x20000), INVALID), (dict(top_logprob=0x50010), INVALID),
    (dict(top_tokens=0x10000), INVALID), (dict(logprob=0x60020), INVALID), (dict(value_type=3), INVALID), (dict(value_type=-1), INVALID),
    (dict(rows=1 << 31), INVALID), (dict(vocabulary=1 << 31), INVALID), (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID), (dict(scale=float("nan")), INVALID),
    (dict(scale=float("inf")), INVALID), (dict(scale=1e-31), INVALID), (dict(scale=2e30), INVALID), (dict(tokens=ODD), INVALID), (dict(logprob=ODD), INVALID),
    (dict(entropy=ODD), INVALID), (dict(lse=ODD), INVALID), (dict(top_tokens=NULL), INVALID), (dict(top_tokens=ODD), INVALID), (dict(top_logprob=NULL), INVALID),
    (dict(top_logprob=ODD), INVALID), (dict(status=NULL), INVALID), (dict(status=ODD), INVALID), (dict(ws=NULL), INVALID), (dict(ws=FAKE + 16), INVALID),
    (dict(ws_bytes=16), SMALL), (dict(n_top=33), UNSUPPORTED), (dict(rows=1 << 24), UNSUPPORTED), (dict(rows=0, logits=NULL, ws=NULL), OK)])
def test_token_scores(change, want):
    assert scores(**change) == want


def test_token_scores_workspace():
    f = binding.fikit_token_scores_workspace_bytes
    assert f(1, 131072, 0, 20) > 0 and f(1, 131072, 2, 32) > f(1, 131072, 2, 0) > 0
    assert f(1, 131072, 0, 33) == f(1 << 24, 10, 0, 3) == f(1, 10, 3, 3) == f(1, 10, 0, 3) == f(100000, 131072, 0, 20) == 0


def test_token_scores_binding():
    x, t, status, native = torch.zeros(3, 10), torch.zeros(3, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), binding._marshal()

    def call(logits=x, tokens=t, n_top=2, out=None):
        return native.token_scores(logits, tokens, status, 1.0, n_top, out, None, 0)
    with pytest.raises(ValueError):
        binding.fikit_token_scores(x, t, status)                             # tensors on a GPU
    f = torch.zeros(3)
    for bad in (dict(logits=x.double()), dict(logits=x[0]), dict(logits=x.t()), dict(tokens=t[:2]), dict(tokens=t.long()), dict(logits=x.clone().requires_grad_()),
                dict(n_top=-1), dict(out=(f, f, f)), dict(out=(f, f, f, None, None)), dict(out=(f[:2], f, f, x[:, :2].int(), x[:, :2])),
                dict(out=(f, f, f, x[:, :2].contiguous(), x[:, :2].contiguous()))):
        with pytest.raises(ValueError):
            call(**bad)
    assert call(n_top=33) == UNSUPPORTED and call(logits=x[:0], tokens=t[:0])[0].shape == (0,)
