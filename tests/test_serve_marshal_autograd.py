"""What the marshalling of a service's calls owes to torch's bookkeeping of gradients, without a GPU: tangents, outputs, versions."""
import ctypes

import pytest
import torch
import torch.autograd.forward_ad as forward_ad

from paper_2311_10359_amd import binding
from test_serve_marshal import address, append, cache, decode, i32, marshal, nothing, prompt, vectors  # noqa: F401

AROUND = ("fikit_rotate_heads", "fikit_cache_fork_workspace_bytes", "fikit_cache_fork", "fikit_cache_compact_workspace_bytes", "fikit_cache_compact",
          "fikit_cache_copy", "fikit_token_scores_workspace_bytes", "fikit_token_scores")


def scores(logits):
    return binding._marshal().token_scores(logits, None, i32(1), 1.0, 0, None, None, 0)


def rotate(q=None, k=None, weight=None, frequencies=None, out=None):
    """Of no tokens, so that nothing is enqueued."""
    x = vectors(rows=0)
    return binding._marshal().rotate_heads(x if q is None else q, x if k is None else k, i32(0), frequencies, i32(1), weight, None, 1e-6, False, out, 0)


def test_inputs_with_a_tangent_are_refused(marshal):  # noqa: F811
    """A dual tensor's output would have none, without a word."""
    native = marshal(nothing)

    def dual(t):
        return forward_ad.make_dual(t, torch.ones_like(t))
    with forward_ad.dual_level():
        x, none = dual(vectors()), dual(vectors(rows=0))
        for call in (lambda: decode(native, q=x), lambda: prompt(native, q=x), lambda: prompt(native, k=x), lambda: prompt(native, v=x),
                     lambda: append(native, k=x), lambda: append(native, v=x), lambda: scores(dual(torch.zeros(0, 10))), lambda: rotate(q=none),
                     lambda: rotate(k=none), lambda: rotate(weight=dual(torch.ones(64, dtype=torch.bfloat16))), lambda: rotate(frequencies=dual(torch.ones(16)))):
            with pytest.raises(ValueError, match="tangent"):
                call()
        decode(native, q=forward_ad.unpack_dual(x).primal)
        assert scores(torch.zeros(0, 10))[2].shape == (0,) and rotate()[0].shape == (0, 2, 64)


def test_gradients_that_are_off_do_not_hide_a_tangent(marshal):  # noqa: F811
    """no_grad() is about reverse mode; forward mode goes on in it."""
    native = marshal(nothing)
    with forward_ad.dual_level(), torch.no_grad():
        x = forward_ad.make_dual(vectors(), torch.ones_like(vectors()))
        with pytest.raises(ValueError, match="tangent"):
            decode(native, q=x)
        with torch.inference_mode():                   # (and not in this)
            decode(native, q=x)


@pytest.fixture
def replaced(marshal):  # noqa: F811
    """The module, with a C function in the place of all that enqueue."""
    def replace(f):
        native = marshal(f)
        native.bind_around(*(address(getattr(binding.load(), name) if "bytes" in name else f) for name in AROUND))
        return native
    return replace


def outputs(floating):
    """Calls into given outputs: (name, function of the module and outputs, those outputs)."""
    x, table, codes = vectors(), i32(3, 2), cache()
    flat = [torch.zeros(3), torch.zeros(3), torch.zeros(3), i32(3, 2), torch.zeros(3, 2)]
    tensors = [
        ("decode", lambda n, o: n.cache_attention(*codes, x, table, i32(3), 0.1, i32(1), None, True, tuple(o), None, 0), [vectors(), torch.zeros(3, 2)]),
        ("prompt", lambda n, o: n.prompt_attention(x, x, x, i32(2), 0.1, i32(1), True, tuple(o), 0), [vectors(), torch.zeros(3, 2)]),
        ("rotate", lambda n, o: n.rotate_heads(x, x, i32(3), None, i32(1), None, None, 1e-6, False, tuple(o), 0), [vectors(), vectors()]),
        ("scores", lambda n, o: n.token_scores(torch.zeros(3, 10), i32(3), i32(1), 1.0, 2, tuple(o), None, 0), flat)]
    if floating:
        return tensors
    return tensors + [
        ("plan", lambda n, o: n.cache_plan(i32(3), i32(3), 5, 16, o[0], i32(6), i32(1), True, tuple(o[1:]), None, 0),
         [i32(3, 4), i32(3), i32(4), torch.zeros(5, dtype=torch.int64), i32(binding.fikit_cache_pieces(5, 3, 16), 4), i32(2)]),
        ("append", lambda n, o: n.cache_append(*o, x, x, i32(2, 4), i32(1), 0), list(cache())),
        ("fork", lambda n, o: n.cache_fork(table, i32(3), i32(5), 16, 9, i32(4), i32(1), tuple(o), None, 0), [i32(5, 2), i32(5), i32(5, 2), i32(9), i32(3)]),
        ("compact", lambda n, o: n.cache_compact(table, i32(3), 16, 9, i32(4), i32(1), tuple(o), None, 0), [i32(3, 2), i32(4, 2), i32(4), i32(2)]),
        ("copy", lambda n, o: n.cache_copy([o[:4], o[4:]], i32(2, 2), i32(1), 0), [*cache(), *cache()])]


def test_outputs_that_require_gradients_are_refused(replaced):
    """They would be written without a trace of where their values come from."""
    native = replaced(nothing)
    for name, call, out in outputs(floating=True):
        for i, t in enumerate(out):
            if t.is_floating_point():
                changed = list(out)
                changed[i] = t.clone().requires_grad_()
                with pytest.raises(ValueError, match="no_grad"):
                    call(native, changed)
                with torch.no_grad():
                    call(native, changed)
                with forward_ad.dual_level(), pytest.raises(ValueError, match="tangent"):
                    changed[i] = forward_ad.make_dual(t.clone(), torch.ones_like(t))
                    call(native, changed)


def test_what_is_written_in_place_has_another_version(replaced):
    """... each tensor that a call writes, none that it reads; of its own outputs a call needs none."""
    native = replaced(nothing)
    for name, call, out in outputs(floating=False):
        before = [t._version for t in out]
        call(native, out)
        assert all(t._version > v for t, v in zip(out, before)), name
    x, logits = vectors(), torch.zeros(3, 10)
    native.rotate_heads(x, x, i32(3), None, i32(1), None, None, 1e-6, False, None, 0)
    prompt(native, q=x)
    native.token_scores(logits, None, i32(1), 1.0, 0, None, None, 0)
    assert x._version == 0 and logits._version == 0
    native.rotate_heads(x, None, i32(3), None, i32(1), None, None, 1e-6, False, (x, None), 0)
    assert x._version == 1


def test_outputs_of_a_call_go_into_the_next(replaced):
    """They are parts of one piece of memory."""
    native, logits = replaced(nothing), torch.zeros(3, 10)
    for mode in (torch.enable_grad, torch.inference_mode):
        with mode():
            out = native.token_scores(logits, i32(3), i32(1), 1.0, 2, None, None, 0)
            native.token_scores(logits, i32(3), i32(1), 1.0, 2, out, None, 0)
        assert all(t.is_inference() or t._version == 1 for t in out) and all(t.is_inference() == (mode is torch.inference_mode) for t in out)
        native.token_scores(logits, i32(3), i32(1), 1.0, 2, out, None, 0)


def test_what_a_refused_call_has_not_written_keeps_its_version(replaced):
    @ctypes.CFUNCTYPE(ctypes.c_int)
    def refused():
        return binding.FIKIT_INVALID_ARG
    native = replaced(refused)
    for name, call, out in outputs(floating=False):
        assert call(native, out) == binding.FIKIT_INVALID_ARG and all(t._version == 0 for t in out), name


def test_a_backward_pass_notices(replaced):
    """Heads that a product has saved are rotated in place: its backward pass would use other values."""
    native = replaced(nothing)
    q, w = vectors().float(), torch.ones(64, requires_grad=True)
    heads = q.to(torch.bfloat16)
    y = (heads * w).sum()
    native.rotate_heads(heads[:, :1], None, i32(3), None, i32(1), None, None, 1e-6, False, (heads[:, :1], None), 0)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()


def test_inference_tensors_have_no_version(replaced):
    native = replaced(nothing)
    with torch.inference_mode():
        made = outputs(floating=False)
        for _, call, out in made:
            call(native, out)
    for _, call, out in made:
        call(native, out)
