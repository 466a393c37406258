"""Host-side test of the streams that calls with adapters and norms take."""
from __future__ import annotations

import types

import pytest
import torch

from paper_2606_11244_amd import spear as sp


def test_a_stream_of_another_device_is_refused():
    """The tensors' kernels may not run on another GPU."""
    def stream(i):
        return types.SimpleNamespace(device=torch.device("cuda", i), cuda_stream=64 + i)
    assert sp._raw_stream(stream(0), 0) == 64 and sp._raw_stream(stream(3), 3) == 67
    for i, dev in ((1, 0), (0, 2)):
        with pytest.raises(ValueError, match="device"):
            sp._raw_stream(stream(i), dev)
