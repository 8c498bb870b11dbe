"""Page tables whose entries are more than int32 counts."""
import pytest
import torch

import paper_2205_10034_amd as M

pytestmark = pytest.mark.gpu


def test_reserve_in_a_table_of_more_than_2_31_entries():
    """1024 sequences of 2^21 + 1 pages of one place, 8.6 GB of entries; a hundred pages are free, and go to the first sequence."""
    S, W, N = 1024, 2 ** 21 + 1, 120
    k = torch.zeros(N, 1, 1, 8, dtype=torch.bfloat16, device="cuda")
    table = torch.full((S, W), -1, dtype=torch.int32, device="cuda")
    cache = M.KVCache(k, torch.zeros_like(k), table)
    refs = torch.zeros(N, dtype=torch.int32, device="cuda")
    refs[::6] = 1                                            # 20 are in use (by nobody here)
    free = torch.nonzero(refs == 0)[:, 0].int()
    lens = torch.full((S,), W, dtype=torch.int32, device="cuda")
    ws, missing = torch.empty(M.moe_kv_pages_workspace_bytes(cache), dtype=torch.uint8, device="cuda"), torch.full((1,), -5, dtype=torch.int32, device="cuda")
    M.moe_kv_reserve(cache, refs, lens, ws, missing=missing)
    torch.cuda.synchronize()
    assert missing.item() == 2 ** 31 - 1 and S * W - 100 > 2 ** 31 - 1
    assert torch.equal(table[0, :100], free) and (refs == 1).all()
    table[0, :100] = -1
    assert all(bool((table[s:s + 64] == -1).all()) for s in range(0, S, 64))
    # fewer than 2^31 are wanted, though the sequences' sum passes it before the last ones
    lens[:] = torch.tensor([W] * 1023 + [0], dtype=torch.int32)
    refs.zero_()
    refs[7:] = 1
    M.moe_kv_reserve(cache, refs, lens, ws, missing=missing)
    torch.cuda.synchronize()
    assert missing.item() == 1023 * W - 7 and torch.equal(table[0, :8].cpu(), torch.tensor([0, 1, 2, 3, 4, 5, 6, -1], dtype=torch.int32))
