"""The compiled marshalling of the attention calls, without a GPU: the C calls are replaced, tensors lie in host memory."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2311_10359_amd import binding

NAMES = ("fikit_cache_pieces", "fikit_cache_plan_workspace_bytes", "fikit_cache_plan", "fikit_cache_append",
         "fikit_cache_attention_workspace_bytes", "fikit_cache_attention", "fikit_prompt_attention")
CALLS = ("fikit_cache_plan", "fikit_cache_append", "fikit_cache_attention", "fikit_prompt_attention")


def address(f):
    return ctypes.cast(f, ctypes.c_void_p).value


@pytest.fixture
def marshal():
    """The module, and a function that puts another C function in the place of the four calls."""
    native = binding._marshal()

    def replace(f):
        native.bind(*(address(f if name in CALLS else getattr(binding.load(), name)) for name in NAMES))
        return native
    yield replace
    binding._native = None
    binding._marshal()


nothing = ctypes.CFUNCTYPE(ctypes.c_int)(lambda: 0)


def i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def vectors(rows=3, heads=2, dim=64):
    return torch.zeros((rows, heads, dim), dtype=torch.bfloat16)


def cache():
    codes, exps = torch.zeros((4, 2, 16, 64), dtype=torch.uint8), torch.ones((4, 2), dtype=torch.uint8)
    return codes, codes.clone(), exps, exps.clone()


def plan(native, want_slots=True):
    return native.cache_plan(i32(3), i32(3), 5, 16, i32(3, 4), i32(6), i32(1), want_slots, None, None, 0)


def append(native, k=None, v=None):
    return native.cache_append(*cache(), vectors() if k is None else k, vectors() if v is None else v, i32(2, 4), i32(1), 0)


def decode(native, q=None, want_lse=True):
    return native.cache_attention(*cache(), vectors() if q is None else q, i32(3, 2), i32(3), 0.1, i32(1), None, want_lse, None, None, 0)


def prompt(native, q=None, k=None, v=None, want_lse=True):
    q = vectors() if q is None else q
    k, v = (torch.zeros_like(q, requires_grad=False) if x is None else x for x in (k, v))
    return native.prompt_attention(q, k, v, i32(2), 0.1, i32(1), want_lse, None, 0)


@pytest.mark.parametrize("want", [True, 1, np.True_, False, 0, np.False_, None])
def test_wanted_outputs_go_by_truth(marshal, want):
    native = marshal(nothing)
    assert (plan(native, want)[2] is not None) == bool(want)
    assert (decode(native, want_lse=want)[1] is not None) == bool(want)
    assert (prompt(native, want_lse=want)[1] is not None) == bool(want)


def test_the_interpreter_is_free_while_a_call_enqueues(marshal):
    """PyGILState_Check, called in the place of the C calls, tells whether the calling thread holds the interpreter's lock."""
    native = marshal(ctypes.pythonapi.PyGILState_Check)
    assert isinstance(plan(native), tuple) and isinstance(decode(native), tuple) and isinstance(prompt(native), tuple)
    assert append(native) == 0


def test_inputs_that_require_gradients_are_refused(marshal):
    """Their outputs would be cut off from them without a word; there is no backward pass."""
    native = marshal(nothing)
    x = vectors().requires_grad_()
    for call in (lambda: decode(native, q=x), lambda: prompt(native, q=x), lambda: prompt(native, k=x), lambda: prompt(native, v=x),
                 lambda: append(native, k=x), lambda: append(native, v=x)):
        with pytest.raises(ValueError, match="no_grad"):
            call()
        with torch.no_grad():
            call()
    decode(native, q=x.detach())


def test_strides_of_single_tokens_and_heads_do_not_count(marshal):
    """What a dimension of size one has for a stride is chance: a slice's, say, that is no multiple of 8 values."""
    seen = []

    @ctypes.CFUNCTYPE(ctypes.c_int, ctypes.POINTER(binding._Vectors), ctypes.POINTER(binding._Vectors), ctypes.POINTER(binding._Vectors))
    def prompt_attention(q, k, v):
        seen.extend((x.contents.token_stride, x.contents.head_stride) for x in (q, k, v))
        return 0
    native = marshal(prompt_attention)
    one_token = torch.as_strided(torch.zeros(1024, dtype=torch.bfloat16), (1, 2, 64), (17, 64, 1))
    prompt(native, q=one_token, k=one_token, v=one_token)
    one_head = torch.as_strided(torch.zeros(1024, dtype=torch.bfloat16), (3, 1, 64), (72, 3, 1))
    prompt(native, q=one_head, k=one_head, v=one_head)
    assert seen == [(0, 64)] * 3 + [(72, 0)] * 3
