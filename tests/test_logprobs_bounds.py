"""Host-only: the bounds of the log-probabilities' tests let nothing through that is wrong by more than rounding."""
import numpy as np
import pytest

from logprobs_util import Rows, confident
from oracle import drafts_oracle as O


def rounded(x, dtype="f32"):
    if dtype == "f32":
        return np.float32(x)
    import torch
    return torch.from_numpy(np.asarray(x)).bfloat16().float().numpy()


def forward_of(h, ids, scale):
    logp, lse, entropy, *_ = O.logprobs(h, ids, scale)
    return dict(logp=rounded(logp), lse=rounded(lse), entropy=rounded(entropy))


@pytest.mark.parametrize("V", [2, 700, 50001, 262145])
def test_results_that_are_off(V):
    rng = np.random.default_rng(V)
    h, ids = np.float32(3 * rng.standard_normal((3, V))), rng.integers(0, V, 3)
    rows, got = Rows(h, ids, 1.3), forward_of(h, ids, 1.3)
    rows.check_forward(got)
    for name in got:
        for by in (5e-5, -5e-5):
            with pytest.raises(AssertionError, match=name):
                rows.check_forward({**got, name: got[name] + np.float32(by)})


@pytest.mark.parametrize("dtype,slightly", [("f32", 1.001), ("bf16", 1.02)])
@pytest.mark.parametrize("V", [2, 700, 50001, 262145])
def test_gradients_that_are_off(V, dtype, slightly):
    rng = np.random.default_rng(V)
    h, ids = rounded(3 * rng.standard_normal((2, V)), dtype), rng.integers(0, V, 2)
    rows = Rows(h, ids, 0.8)
    for g in (dict(d_logp=[1.0, -2.0]), dict(d_entropy=[0.5, 1.0]), dict(d_lse=[1.0, 0.1]), dict(d_logp=[1.0, 0.0], d_entropy=[0.0, 0.7], d_lse=[0.3, 0.3])):
        want, _ = O.logprobs_gradient(h, ids, 0.8, **g)
        rows.check_gradient(rounded(want, dtype), dtype, **g)
        with pytest.raises(AssertionError):
            rows.check_gradient(rounded(want * slightly, dtype), dtype, **g)


@pytest.mark.parametrize("dtype,level", [("f32", 0.0), ("f32", 60.0), ("f32", 100.0), ("bf16", 0.0), ("bf16", 250.0), ("bf16", 1000.0)])
@pytest.mark.parametrize("left", [1e-2, 1e-4, 4e-6])
def test_own_gradient_of_a_confident_row(left, dtype, level):
    """1 - p taken as a difference, from p = exp(x - lse) with lse one rounded number, is not near enough; nor is 0."""
    h, ids = confident(4, 5000, dtype, level, left)
    rows = Rows(h, ids)
    want, _ = O.logprobs_gradient(h, ids, 1.0, np.ones(4))
    t = np.arange(4)
    exact = [np.exp(np.delete(np.float64(h[i]), ids[i]) - rows.lse[i]).sum() for i in range(4)]
    assert np.allclose(want[t, ids], exact, rtol=1e-6)
    rows.check_gradient(rounded(want, dtype), dtype, d_logp=np.ones(4))
    wrong = want.copy()
    wrong[t, ids] = 0.0
    with pytest.raises(AssertionError, match="4 off"):
        rows.check_gradient(rounded(wrong, dtype), dtype, d_logp=np.ones(4))
    if level * 2.0 ** -24 > left * (0.02 if dtype == "bf16" else 1e-3):
        wrong[t, ids] = 1 - np.exp(np.float32(h[t, ids]) - np.float64(rounded(rows.lse) * (1 + 2.0 ** -25)))   # (half of what rounding can do)
        with pytest.raises(AssertionError):
            rows.check_gradient(rounded(wrong, dtype), dtype, d_logp=np.ones(4))
