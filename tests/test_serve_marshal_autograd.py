"""What the marshalling of a service's calls owes to torch's bookkeeping of gradients, without a GPU: tangents of forward mode."""
import pytest
import torch
import torch.autograd.forward_ad as forward_ad

from paper_2311_10359_amd import binding
from test_serve_marshal import append, decode, i32, marshal, nothing, prompt, vectors  # noqa: F401


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
