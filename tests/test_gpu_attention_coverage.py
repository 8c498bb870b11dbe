"""Every kept place enters the decode attention once: long splits, ragged batches, windows."""
import numpy as np
import pytest

from attention_coverage import Marked

pytestmark = pytest.mark.gpu

RAGGED = np.random.default_rng(3).integers(0, 6000, 60).tolist()
LENS = {"long": [70001], "longest": [131071, 5, 0, 9000], "split": [20000, 1, 4097, 0, 513, 20000], "ragged": RAGGED, "one part more": [1025] * 33,
        "many": [40, 0, 1, 700] * 130, "many, one long": [17] * 300 + [12345] + [0] * 300}
ALL_LENGTHS = sorted(set(n for lens in LENS.values() for n in lens if n))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,D", [(8, 2, 64), (1, 1, 128), (12, 4, 128), (40, 2, 256), (64, 1, 64), (3, 3, 64)])
@pytest.mark.parametrize("lens", LENS.values(), ids=LENS.keys())
def test_every_place_once(lens, hq, hkv, D, dtype):
    print(len(lens), hq, hkv, D, dtype, flush=True)
    m = Marked(lens, hkv, D, 16, dtype)
    m.check(hq)
    m.check(hq, window=1500)
