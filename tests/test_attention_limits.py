"""Host-only checks of the attention half's limits: calls that no launch can do are refused before the first one."""
import ctypes as C

import pytest
import torch

import paper_2205_10034_amd as M
from paper_2205_10034_amd import attention as B
from test_attention_abi import FAKE, OPT, ROWS, cache, compiled, rotary

UNSUPPORTED = 2


@pytest.mark.parametrize("kw,hq,window", [
    (dict(n_seqs=2 ** 31 - 1, table_width=1), 2, 0),                 # whole sequences, a workgroup each
    (dict(n_seqs=2 ** 24, table_width=1), 2, 0),                     # 2^24 workgroups: 2^32 work-items, one too many
    (dict(n_seqs=2 ** 24, table_width=16, n_kv_heads=1), 64, 0),     # sequences of up to 256 places, four tiles of heads: the same
    (dict(n_seqs=2 ** 25, table_width=100), 2, 0),                   # sequences that are split: 2^26 rows to join
    (dict(n_seqs=2 ** 20, table_width=100, n_kv_heads=64), 64, 0),
    (dict(n_seqs=2 ** 25, table_width=100), 2, 4000),
    (dict(n_seqs=2 ** 25, table_width=100), 2, 16),                  # whole by the window
])
def test_attention_refuses_what_no_launch_can_do(kw, hq, window):
    L, c, x = B.lib(), cache(**kw), ROWS()
    opt = OPT(window=window)
    assert L.moe_attention_decode(C.byref(c), hq, C.byref(x), FAKE, C.byref(opt), C.byref(x), None, FAKE, 1 << 60, None) == UNSUPPORTED
    assert b"too many" in L.moe_last_error()


@pytest.mark.parametrize("T", [2 ** 26 - 3, 2 ** 26, 2 ** 31 - 1])
def test_rotary_and_append_refuse_what_no_launch_can_do(T):
    """Four tokens a workgroup of 256: 2^26 - 4 tokens are the most."""
    L, r, x, y, c = B.lib(), rotary(), ROWS(), ROWS(FAKE * 2), cache()
    assert L.moe_rotary(C.byref(r), 1, T, 2, C.byref(x), FAKE, C.byref(y), 0, None) == UNSUPPORTED and b"too many" in L.moe_last_error()
    assert L.moe_kv_append(C.byref(c), T, C.byref(x), C.byref(x), FAKE, FAKE, C.byref(r), FAKE, 2, C.byref(x), C.byref(y), None) == UNSUPPORTED


def test_what_a_launch_can_do_on_the_host(tmp_path):
    compiled(tmp_path, """int main() {
  assert(launchable(1, 256) && launchable((1 << 24) - 1, 256) && !launchable(1 << 24, 256) && !launchable(1ll << 40, 256));
  assert(launchable(4294967295ll, 1) && !launchable(4294967296ll, 1) && !launchable(1ll << 31, 256));
}""")


def test_numbers_beyond_32_bits_are_not_cut():
    """What the library takes as int32 is refused by the binding, or kept in meaning, and never loses its upper bits."""
    meta = lambda *shape, dtype=torch.bfloat16: torch.empty(*shape, dtype=dtype, device="meta")
    assert B._int32(2 ** 31 - 1, "n") == 2 ** 31 - 1 and B._int32(-3, "n") == -3
    for n in (2 ** 31, 2 ** 32 + 1, -2 ** 31 - 1):
        with pytest.raises(ValueError, match="int32"):
            B._int32(n, "n")
    # a window longer than any sequence is no window; a negative one stays what the library refuses
    for window, taken in ((0, 0), (5, 5), (2 ** 31 - 1, 2 ** 31 - 1), (2 ** 32 + 1, 2 ** 31 - 1), (2 ** 63 - 1, 2 ** 31 - 1), (-1, -1), (-2 ** 32 + 7, -1)):
        assert B._options(0.5, 1.5, window, None).window == taken
    x = meta(2 ** 32 + 1, 1, 2)
    rot = type("R", (), dict(device=-1, head_dim=2, n_axes=1, c=rotary(head_dim=2, rot_dim=2, pairs=(1,))))
    with pytest.raises(ValueError, match="int32"):
        M.moe_rotary(rot, x, meta(1, 2 ** 32 + 1, dtype=torch.int32), x)
    pool = type("P", (), dict(device=-1, dtype=torch.bfloat16, head_dim=64, n_kv_heads=1, n_seqs=1, c=cache()))
    with pytest.raises(ValueError, match="int32"):
        k = meta(2 ** 32 + 1, 1, 64)
        M.moe_kv_append(pool, k, k, meta(2 ** 32 + 1, dtype=torch.int32))
    with pytest.raises(ValueError, match="int32"):
        M.moe_attention_decode_workspace_bytes(pool, 2 ** 32 + 4)
