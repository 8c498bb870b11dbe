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
