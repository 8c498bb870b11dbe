"""Log-probabilities and their gradient within bounds of each element's own rounding: every division of rows among wavefronts, in place and
not."""
import numpy as np
import pytest

from logprobs_util import Rows
from test_gpu_token_logprobs import backward, forward, ids_for, logits

pytestmark = pytest.mark.gpu

# one wavefront to a row (one chunk of 1024 logits; several), four (some chunks each, or one), sixteen
SHAPES = [(1, 1), (7, 63), (300, 1000), (4099, 2050), (4096, 4001), (500, 2050), (1030, 9001), (300, 20011), (5, 17001), (1, 50001), (3, 262145), (260, 70001)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,V", SHAPES)
def test_forward_and_gradient(T, V, dtype):
    rng = np.random.default_rng(V)
    x, h = logits(T, V, dtype, seed=V, stride=V + 3, offset=5)
    ids = ids_for(T, V)
    some = np.unique(np.r_[:min(T, 40), T - 1])                         # (the oracle's rows)
    rows = Rows(h[some], ids[some], 0.9)
    fwd = forward(x, ids, scale=0.9)
    rows.check_forward({k: v[some] for k, v in fwd.items()})
    g = {n: rng.standard_normal(T).astype(np.float32) for n in ("d_logp", "d_entropy", "d_lse")}
    for names in (("d_logp",), ("d_entropy",), ("d_logp", "d_entropy", "d_lse")):
        mine = {n: g[n] for n in names}
        for in_place in (False, True):
            got = backward(x.clone() if in_place else x, ids, fwd, scale=0.9, stride=V + 1, in_place=in_place, **mine)
            rows.check_gradient(got[some], dtype, **{n: v[some] for n, v in mine.items()})
