"""Host-only: calls of a step of drafted tokens that could not be answered rightly are refused."""
import ctypes as C

import pytest
import torch

from paper_2205_10034_amd import attention as A
from paper_2205_10034_amd import drafts as D
from test_attention_abi import FAKE, cache


@pytest.mark.parametrize("offset", [-2, -1, 0, 1, 2])
def test_new_lengths_over_the_old_ones(offset):
    """A sequence's new length would be written where another workgroup has yet to read a base."""
    c = cache(n_seqs=3)
    assert D.lib().moe_kv_compact(C.byref(c), FAKE, 4, 4 * FAKE, FAKE + 4 * offset, None) == 1
    assert b"overlap" in D.lib().moe_last_error()


class Stream:
    def __init__(self, device_index, cuda_stream):
        self.device_index, self.cuda_stream = device_index, cuda_stream


def test_streams_of_other_devices(monkeypatch):
    """A default stream is the current device's; a call for another device's tensors would run there."""
    handles = {0: 0, 1: 0, 2: 4096}
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: handles[device], raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    assert A._stream(None, 0) is None and A._stream(None, 2) == 4096
    assert A._stream(Stream(0, 0), 0) is None and A._stream(Stream(1, 512), 1) == 512
    with pytest.raises(ValueError, match="current device"):
        A._stream(None, 1)
    with pytest.raises(ValueError, match="current device"):
        A._stream(Stream(1, 0), 1)
    for index, handle in ((1, 512), (0, 0)):
        with pytest.raises(ValueError, match="stream of CUDA device"):
            A._stream(Stream(index, handle), 2)
