"""The binding's choice of streams and the example service's bookkeeping, without a GPU."""
from types import SimpleNamespace

import pytest
import torch

from paper_2311_10359_amd import binding, service

SIZES = service.Sizes(layers=1, q_heads=2, kv_heads=1, dim=64, block=16, blocks=8, vocabulary=16)


def test_a_stream_of_another_device_is_refused():
    """The call would run on the tensors' device, on a stream that nobody named."""
    with pytest.raises(ValueError):
        binding._elsewhere(SimpleNamespace(device=torch.device("cuda", 1)), torch.device("cuda", 0))
