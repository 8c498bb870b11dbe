"""Softmax of the decode attention where its arithmetic shows: outputs that cancel, values and scores near the ends of float32."""
import numpy as np
import pytest
import torch

from attention_util import DT, HALF_STEP, Paged, attend
from oracle import attention_oracle as A

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("bf16", 128), ("bf16", 256), ("f32", 64), ("f32", 256)])
def test_weights_keep_the_bits_of_float32(dtype, D):
    """Three keys with scores a, a + 2^-12 and a + t and values -1, 1 and 0: out = (w1 - w0) / sum w, some 2^-14, lays the weights'
    own errors bare.  Scores are exact, at most 2; every other step of a weight (scale, difference to the maximum, change to powers of
    two) rounds 2^-24 |z| or less each, 6 * 2^-24 together, the power itself is good to 2^-23, the sums of three to 2 * 2^-24: at most
    10 * 2^-24 of a weighted mean of |v| that is below 1.  Then one rounding."""
    S = 96
    p = Paged([3] * S, 1, D, 4, dtype)
    rng = np.random.default_rng(7)
    a, t = rng.integers(0, 128, S) / 128.0, rng.integers(1, 128, S) / 128.0
    p.k[p.table[:, 0], :3] = p.v[p.table[:, 0], :3] = 0.0
    page = p.table[:, 0]
    p.k[page, :3, 0, 0] = a[:, None]
    p.k[page, 1, 0, 1], p.k[page, 2, 0, 1] = 2.0 ** -12, t
    p.v[page, 0], p.v[page, 1] = -1.0, 1.0
    q = torch.zeros(S, 2, D)
    q[:, :, :2] = 1.0
    q = q.to(DT[dtype])
    out, lse = attend(p.cache(), q, p.lens, scale=1.0)
    ref, ref_lse, mean_abs, *_ = A.decode(p.k, p.v, p.table, q.float().numpy(), p.lens, 1.0)
    off, tol = np.abs(out - ref), 10 * 2.0 ** -24 * mean_abs + HALF_STEP[dtype] * 1.01 * np.abs(ref)
    assert (off <= tol).all(), f"{(off > tol).sum()} of {off.size} off, by up to {(off / tol).max():.1f} times what is allowed"
    assert np.abs(lse - ref_lse).max() <= 16 * 2.0 ** -24 * 4


@pytest.mark.parametrize("dtype,D,far", [("bf16", 64, 128), ("bf16", 256, 64), ("f32", 64, 64), ("f32", 256, 64)])
def test_large_values_under_rising_scores(dtype, D, far):
    """Values near the type's largest whose keys are a little better than those before them: the mean of finite values is finite.
    All scores are equal but one, 5.4 higher (a factor of 222), in place `far`, a tile that the same wavefront takes later.  Scores
    are exact and below 6, so weights are off by 64 * 2^-24 at most (scale, differences, exponent on |z| < 8, the power), sums of
    n by n * 2^-24."""
    lens = [129, 200, 257, 1000, 3000]
    p = Paged(lens, 1, D, 16, dtype)
    big = torch.tensor(3e38).to(DT[dtype]).item()
    for s, n in enumerate(lens):
        for i in range(-(-n // 16)):
            rows = min(16, n - i * 16)
            p.k[p.table[s, i], :rows], p.v[p.table[s, i], :rows] = 0.0, 1.0
        at = (p.table[s, far // 16], 0, 0)
        p.k[at][0], p.v[at][:] = 5.40625, big
        p.v[at][1::2] = -big
    q = torch.zeros(len(lens), 3, D)
    q[:, :, 0] = 1.0
    q = q.to(DT[dtype])
    out, lse = attend(p.cache(), q, p.lens, scale=1.0)
    ref, ref_lse, mean_abs, *_ = A.decode(p.k, p.v, p.table, q.float().numpy(), p.lens, 1.0)
    lost = int((~np.isfinite(out)).sum())
    assert lost == 0, f"{lost} of {out.size} are not finite"
    tol = (64 + np.array(lens))[:, None, None] * 2.0 ** -24 * mean_abs + HALF_STEP[dtype] * 1.01 * np.abs(ref)
    assert (np.abs(out - ref) <= tol).all()
    assert (np.abs(lse - ref_lse) <= (64 + np.array(lens))[:, None] * 2.0 ** -24 * 2).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("sign", [-1.0, 1.0])
def test_scores_near_the_largest_number(sign, dtype):
    """Scores of 3e38 either way are numbers, not infinities: equal ones share the weight, the mean of n values is off by (n + 8)
    float32 roundings of the mean of |v| and one of its own.  lse is the score, to a rounding."""
    lens = [1, 40, 300, 2500]
    p = Paged(lens, 2, 64, 16, dtype)
    big = torch.tensor(sign * 3e38).to(DT[dtype]).item()
    held = ~np.isnan(p.k)
    p.k[held] = 0.0
    p.k[..., 0] = np.where(held[..., 0], big, np.nan)
    q = torch.zeros(4, 4, 64)
    q[:, :, 0] = 1.0
    for kw in (dict(scale=1.0), dict(scale=1.0, window=17)):
        out, lse = attend(p.cache(), q.to(DT[dtype]), p.lens, **kw)
        ref, ref_lse, mean_abs, *_ = A.decode(p.k, p.v, p.table, q.numpy(), p.lens, **kw)
        tol = (np.array(lens) + 8)[:, None, None] * 2.0 ** -24 * mean_abs + HALF_STEP[dtype] * 1.01 * np.abs(ref)
        off = ~(np.abs(out - ref) <= tol)
        assert not off.any(), f"{off.sum()} of {off.size} off: {out[off][:4]} for {ref[off][:4]}"
        assert (np.abs(lse / ref_lse - 1.0) <= 2.0 ** -23).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_smallest_caps(dtype):
    """A cap whose reciprocal float32 does not hold leaves scores of nearly nothing: all places weigh the same, 0 scores included."""
    lens = [3, 70]
    p = Paged(lens, 1, 64, 16, dtype)
    q = torch.zeros(2, 2, 64)
    q[:, 1] = 3.0
    for cap in (1e-45, 1e-39, 1.2e-38, 1e-30):
        out, lse = attend(p.cache(), q.to(DT[dtype]), p.lens, softcap=cap)
        ref, ref_lse, mean_abs, *_ = A.decode(p.k, p.v, p.table, q.numpy(), p.lens, 0.125, softcap=cap)
        tol = (np.array(lens) + 8)[:, None, None] * 2.0 ** -24 * mean_abs + HALF_STEP[dtype] * 1.01 * np.abs(ref)
        off = int((~(np.abs(out - ref) <= tol)).sum())
        assert off == 0, f"cap {cap}: {off} of {out.size} off"
        assert np.abs(lse - ref_lse).max() <= 8 * 2.0 ** -24 * 5
