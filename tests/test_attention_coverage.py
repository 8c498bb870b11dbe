"""The coverage check itself, on the CPU: exact results pass, a lost, doubled or exchanged tile does not, at every length that the GPU
tests use."""
import numpy as np
import pytest
import torch

from attention_coverage import BLOCK, accepted, counts, kept_places
from attention_util import DT
from test_gpu_attention_coverage import ALL_LENGTHS


def result(taken, dtype):
    n = taken.sum()
    if n == 0:
        return np.zeros((1, len(taken))), np.array([-np.inf])
    out = torch.from_numpy((taken / n).astype(np.float32)).to(DT[dtype]).double().numpy()[None]
    return out, np.array([np.log(n)], dtype=np.float32).astype(np.float64)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("n", ALL_LENGTHS)
def test_mistakes_are_seen(n, D, dtype):
    right = counts(np.arange(n), D)
    assert accepted(*result(right, dtype), right, D, dtype)
    tiles = max(1, n // BLOCK)
    for t in {0, 1, tiles // 2, tiles - 1}:
        tile = counts(np.arange(t * BLOCK, min(n, (t + 1) * BLOCK)), D)
        other = counts(np.arange(t * BLOCK, min(n, (t + 1) * BLOCK)) + BLOCK, D)
        if not tile.any():
            continue
        for wrong in (right - tile, right + tile, right - 0.5 * tile, right + tile / tile.max(), right + tile - other, right - tile + other):
            if (wrong >= 0).all() and wrong.sum() > 0:
                assert not accepted(*result(wrong, dtype), right, D, dtype), (t, wrong.sum(), right.sum())


def test_kept_places():
    assert kept_places(10, 0, [], 4).tolist() == list(range(10)) and kept_places(10, 3, [], 4).tolist() == [7, 8, 9]
    assert kept_places(10, 0, [1], 4).tolist() == [0, 1, 2, 3, 8, 9] and kept_places(0, 5, [], 4).size == 0
