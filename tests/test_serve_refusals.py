"""What the attention calls refuse on the host, before any HIP call; pointers are never followed here."""
import ctypes

import pytest
import torch

import serve_model as model
from paper_2311_10359_amd import binding

FAKE, ODD, NULL = 0x10000, 0x10001, None
OK, INVALID, SMALL, UNSUPPORTED = 0, binding.FIKIT_INVALID_ARG, binding.FIKIT_WORKSPACE_TOO_SMALL, binding.FIKIT_UNSUPPORTED


def plan(**change):
    a = dict(cached=FAKE, added=FAKE, n_requests=4, n_tokens=9, block=16, table=FAKE, width=3, free=FAKE, n_free=5, lengths=FAKE, offsets=FAKE,
             slots=FAKE, pieces=FAKE, counts=FAKE, status=FAKE, ws=FAKE, ws_bytes=1 << 20)
    assert set(change) <= set(a)
    a.update(change)
    return binding.load().fikit_cache_plan(*a.values(), None)


@pytest.mark.parametrize("change, want", [
    (dict(cached=NULL), INVALID), (dict(added=ODD), INVALID), (dict(table=NULL), INVALID), (dict(width=0), INVALID), (dict(free=NULL), INVALID),
    (dict(lengths=NULL), INVALID), (dict(offsets=NULL), INVALID), (dict(slots=FAKE + 4), INVALID), (dict(pieces=NULL), INVALID),
    (dict(pieces=FAKE + 8), INVALID), (dict(counts=NULL), INVALID), (dict(status=NULL), INVALID),
    (dict(n_requests=20000, ws=NULL), INVALID), (dict(n_requests=20000, ws=FAKE + 16), INVALID),
    (dict(n_requests=0), INVALID), (dict(n_tokens=1 << 31), INVALID), (dict(n_requests=20000, ws_bytes=16), SMALL), (dict(n_requests=(1 << 20) + 1), UNSUPPORTED),
    (dict(block=0), UNSUPPORTED), (dict(block=8), UNSUPPORTED), (dict(block=48), UNSUPPORTED), (dict(block=512), UNSUPPORTED),
])
def test_plan(change, want):
    assert plan(**change) == want


def cache(**change):
    a = dict(k=FAKE, v=FAKE, k_exp=FAKE, v_exp=FAKE, n_blocks=10, kv_heads=2, block_tokens=16, head_dim=64)
    assert set(change) <= set(a)
    a.update(change)
    return binding._Cache(*a.values())


def vectors(data=FAKE, token=128, head=64):
    return binding._Vectors(data, token, head)


CACHES = [(dict(k=NULL), INVALID), (dict(v=ODD), INVALID), (dict(k_exp=NULL), INVALID), (dict(n_blocks=0), INVALID), (dict(kv_heads=0), INVALID),
          (dict(block_tokens=24), UNSUPPORTED), (dict(block_tokens=8), UNSUPPORTED), (dict(head_dim=96), UNSUPPORTED), (dict(head_dim=256), UNSUPPORTED)]


def append(c=None, k=None, v=None, n_tokens=5, value_type=0, pieces=FAKE, n_pieces=3, status=FAKE):
    return binding.load().fikit_cache_append(c or cache(), k or vectors(), v or vectors(), n_tokens, value_type, pieces, n_pieces, status, None)


def test_append():
    for change, want in CACHES:
        assert append(c=cache(**change)) == want
    for bad in (vectors(NULL), vectors(FAKE + 8), vectors(token=4), vectors(head=68)):
        assert append(k=bad) == INVALID and append(v=bad) == INVALID
    assert append(value_type=2) == INVALID and append(value_type=-1) == INVALID
    assert append(pieces=NULL) == INVALID and append(pieces=FAKE + 4) == INVALID and append(status=NULL) == INVALID
    assert append(n_pieces=1 << 31) == INVALID
    assert append(n_pieces=0, pieces=NULL, k=vectors(NULL)) == OK
    assert binding.load().fikit_cache_append(None, vectors(), vectors(), 5, 0, FAKE, 3, FAKE, None) == INVALID


def attend(c=None, q=None, q_heads=4, value_type=0, table=FAKE, width=8, lengths=FAKE, n=3, longest=128, out=FAKE, lse=FAKE, status=FAKE, ws=FAKE,
           ws_bytes=1 << 30):
    return binding.load().fikit_cache_attention(c or cache(), q or vectors(), q_heads, value_type, 0.1, table, width, lengths, n, longest, out, lse,
                                                status, ws, ws_bytes, None)


def test_cache_attention():
    for change, want in CACHES:
        assert attend(c=cache(**change)) == want
    for bad in (vectors(NULL), vectors(FAKE + 8), vectors(token=4), vectors(head=68)):
        assert attend(q=bad) == INVALID
    assert attend(q_heads=3) == INVALID and attend(q_heads=0) == INVALID and attend(q_heads=1 << 17) == UNSUPPORTED
    assert attend(longest=129) == INVALID and attend(value_type=7) == INVALID
    for change in (dict(table=NULL), dict(lengths=NULL), dict(out=NULL), dict(out=FAKE + 2), dict(lse=ODD), dict(status=NULL)):
        assert attend(**change) == INVALID
    many = dict(n=1, longest=1 << 20, width=1 << 16)
    assert attend(ws_bytes=256, **many) == SMALL and attend(ws=NULL, **many) == INVALID and attend(ws=FAKE + 16, **many) == INVALID
    assert attend(n=0, q=vectors(NULL), lengths=NULL, out=NULL, table=NULL) == OK


def test_prompt_attention():
    def call(q=None, k=None, v=None, q_heads=4, kv_heads=2, dim=64, value_type=0, offsets=FAKE, prompts=2, tokens=9, out=FAKE, lse=FAKE, status=FAKE):
        return binding.load().fikit_prompt_attention(q or vectors(), k or vectors(), v or vectors(), q_heads, kv_heads, dim, value_type, 0.1, offsets,
                                                     prompts, tokens, out, lse, status, None)
    for bad in (vectors(NULL), vectors(FAKE + 8), vectors(token=4), vectors(head=68)):
        assert call(q=bad) == INVALID and call(k=bad) == INVALID and call(v=bad) == INVALID
    assert call(q_heads=3) == INVALID and call(kv_heads=0) == INVALID and call(q_heads=0) == INVALID
    assert call(dim=80) == UNSUPPORTED and call(dim=256) == UNSUPPORTED and call(value_type=2) == INVALID
    for change in (dict(offsets=NULL), dict(out=NULL), dict(out=FAKE + 4), dict(lse=ODD), dict(status=NULL), dict(prompts=0), dict(tokens=1 << 31)):
        assert call(**change) == INVALID
    assert call(tokens=0, prompts=0, q=vectors(NULL), offsets=NULL, out=NULL) == OK


def test_sizes():
    for tokens, requests, block in ((0, 0, 16), (1, 1, 16), (100, 3, 16), (100, 100, 64), (5000, 7, 32)):
        assert binding.fikit_cache_pieces(tokens, requests, block) == model.pieces_room(tokens, requests, block)
    # no cut of the tokens makes more pieces than that
    for cached, added in (([15, 31, 0], [2, 18, 16]), ([15] * 8, [18] * 8), ([0], [1]), ([1, 1], [15, 16])):
        table = [[0] * 9 for _ in cached]
        import numpy as np
        got = model.plan(cached, added, 16, np.array(table), range(99))
        assert got["counts"][1] <= binding.fikit_cache_pieces(sum(added), len(cached), 16)
    lib = binding.load()
    assert lib.fikit_cache_plan_workspace_bytes(1024) == 0 and lib.fikit_cache_plan_workspace_bytes(1025) >= 32
    assert binding.fikit_cache_attention_workspace_bytes(4, 6, 4, 64, 100) == 0
    assert 0 < binding.fikit_cache_attention_workspace_bytes(1, 8, 8, 64, 100) <= binding.fikit_cache_attention_workspace_bytes(1, 8, 8, 128, 100000)
    assert binding.status_string(binding.FIKIT_CACHE_FULL) not in ("ok", "unknown status")


def test_binding_refuses_what_it_cannot_describe():
    x = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    status = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError):
        binding.fikit_prompt_attention(x.float(), x, x, status, 0.1, status)
    with pytest.raises(ValueError):
        binding.fikit_prompt_attention(x.transpose(1, 2), x, x, status, 0.1, status)
    with pytest.raises(ValueError):
        binding.fikit_prompt_attention(x, x[:3], x, status, 0.1, status)
    codes, exps = torch.zeros((3, 2, 16, 64), dtype=torch.uint8), torch.ones((3, 2), dtype=torch.uint8)
    with pytest.raises(ValueError):
        binding.fikit_cache_append(codes, codes[:2], exps, exps, x, x, torch.zeros((1, 4), dtype=torch.int32), status)
    with pytest.raises(ValueError):
        binding.fikit_cache_append(codes, codes, exps[:, :1], exps, x, x, torch.zeros((1, 4), dtype=torch.int32), status)
    with pytest.raises(ValueError):
        binding.fikit_cache_attention(x, codes, codes, exps, exps, torch.zeros((3, 1), dtype=torch.int32), torch.zeros(4, dtype=torch.int32), 0.1, status)


def test_the_model_rounds_as_the_type_does():
    x = torch.cat([torch.linspace(-448, 448, 20001), torch.randn(20000) * 0.01, torch.tensor([0.0, -0.0, 2.0 ** -10, 3 * 2.0 ** -10, -2.0 ** -10])])
    assert (model.round_codes(x.numpy()) == x.to(torch.float8_e4m3fn).view(torch.uint8).numpy()).all()
    for most in (1.0, 448.0, 449.0, 447.0, 3.5, 3.6, 1e30, 1e-37):
        e = model.exponent_for(most)
        assert most <= 448 * 2.0 ** (e - 127) and (e == 1 or most > 448 * 2.0 ** (e - 128))
