"""Tree attention at the end of the longest page table there can be: places up to 2^31 - 3."""
import numpy as np
import pytest
import torch

import paper_2205_10034_amd as M
from attention_util import DT
from drafts_util import attend_tree, check_tree, firsts, tree_words

pytestmark = pytest.mark.gpu


class Far:
    """The last places of one sequence of a table of 42966 pages of 49981 places, all of them one page; as check_tree takes it, moved to the front."""

    WIDTH, PAGE = 42966, 49981

    def __init__(self, kept, D, dtype):
        self.page, self.D, self.dtype, self.n = self.PAGE, D, dtype, kept
        g = torch.Generator().manual_seed(D)
        shape = (1, self.PAGE, 1, D)
        pools = [torch.full(shape, float("nan"), dtype=DT[dtype]) for _ in range(2)]
        for x in pools:
            x[0, -kept:] = torch.randn(kept, 1, D, generator=g).to(DT[dtype])
        self.cache = M.KVCache(*(x.cuda() for x in pools), torch.zeros(1, self.WIDTH, dtype=torch.int32, device="cuda"))
        self.k, self.v = (x[:, -kept:].float().numpy() for x in pools)
        self.table = np.zeros((1, 1), dtype=np.int32)


@pytest.mark.parametrize("D,dtype,n,G", [(64, "bf16", 7, 2), (256, "bf16", 20, 1), (64, "f32", 7, 2), (64, "bf16", 20, 2), (128, "bf16", 40, 2), (256, "bf16", 40, 1)])
@pytest.mark.parametrize("slope", [None, 0.25])
def test_last_places(slope, D, dtype, n, G):
    length, window = Far.WIDTH * Far.PAGE, 100
    assert length == 2 ** 31 - 2
    # (what the window leaves for the deepest token and the shallowest one; distances, and so all scores, are as in a short sequence)
    p = Far(window + n, D, dtype)
    q = (2 * torch.randn(n, G, D, generator=torch.Generator().manual_seed(n))).to(DT[dtype])
    slopes = None if slope is None else np.float32(slope * np.arange(1, G + 1))
    for words in (tree_words([n]), tree_words([n], chain=True), None):
        out, lse = attend_tree(p.cache, q, firsts([n]), [length], n, words, window=window, slopes=slopes)
        check_tree(p, q, firsts([n]), [p.n], n, out, lse, words, window=window, slopes=slopes)
