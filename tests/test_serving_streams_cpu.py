"""The binding's check of a given stream, without a GPU: the serving operators
launch on the tensors' device, which a stream of another one is not on."""
import types

import pytest
import torch

import paper_2605_28803_amd as oq


def _stream(index, handle=0x1234):
    return types.SimpleNamespace(device_index=index, cuda_stream=handle, device=torch.device("cuda", index))


def test_a_stream_of_another_device_is_refused():
    assert oq._on(_stream(0), 0) == 0x1234 and oq._on(_stream(3, 7), 3) == 7
    for index, dev in ((1, 0), (0, 1)):
        with pytest.raises(ValueError, match=f"not on cuda:{dev}"):
            oq._on(_stream(index), dev)
