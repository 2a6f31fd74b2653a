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
    (dict(q_out=vectors(0x30000, token=0)), INVALID), (dict(q_out=vectors(0x30000, head=0)), INVALID),
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
