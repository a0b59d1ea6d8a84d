"""The Python bindings of the operators around the layer step: what they look at before a call.  No GPU needed: nothing is launched."""
import pytest
import torch

from paper_2512_23353_amd import isopo


def test_a_stream_for_host_tensors_is_refused():
    with pytest.raises(ValueError):
        isopo.linear(torch.zeros(4, 16), torch.zeros(8, 16), stream=1)
