"""The gradient of a given token that has nearly all mass, where the entropy counts too:

    dl_t = dlogprob (1 - p) - dentropy p (log p + entropy)

Both terms are small, and neither is what rounding leaves of dlogprob.

Tolerance.  1 - p comes from the log of the sum, which is off by what the weights of the others are: a weight 2^-t by its argument's rounding, t up to 52, so 2^-19
ln 2, and the exponential's own and the sums' few steps of 2^-24; entropy by twice that.  log p + entropy is a sum of two such numbers."""
import numpy as np
import pytest

from tests.lm_ops_util import HALF, U32, rounded
from tests.test_gpu_scores import check_score_gradient, score_gradient

pytestmark = pytest.mark.gpu
WEIGHT = 2.0 ** -19 * np.log(2) + 16 * U32
SUMS = 2 * (1 + 6 + 15) * 2.0 ** -53        # additions in 64 bits behind the 1


def check(l, name, token, dlp, dh):
    M, V = l.shape
    at = np.arange(M)
    d = l - l[at, token][:, None]
    others = np.where(np.arange(V) == token[:, None], 0, np.exp(d))
    rest = others.sum(1)
    far = -(others * np.where(others > 0, d, 0)).sum(1)
    log_p, entropy, p = -np.log1p(rest), np.log1p(rest) + far / (1 + rest), 1 / (1 + rest)
    got = score_gradient(l, name, token, dlp, dh)[at, token]
    want = dlp * rest * p - dh * p * (log_p + entropy)
    size = abs(dlp) * rest * p + abs(dh) * p * (abs(log_p) + entropy)
    assert (abs(got - want) <= 3 * WEIGHT * size + (abs(dlp) + abs(dh)) * SUMS + HALF[name] * abs(want)).all(), (abs(got - want) / size).max()


# a little entropy beside the mean likelihood, as much of both, mostly entropy, entropy alone
WEIGHTS = [(-1 / 700, -0.01 / 700), (1.0, 1.0), (-0.001, 3.0), (0.0, 1.0), (1.0, 0.0)]


@pytest.mark.parametrize("dlp,dh", WEIGHTS)
@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("M,V", [(200, 1000), (1, 10000), (20, 20003)])
def test_sure_tokens(M, V, name, dlp, dh):
    r = np.random.default_rng(V)
    l, token = r.normal(size=(M, V)), r.integers(0, V, M)
    l[np.arange(M), token] = np.log(V) + (np.linspace(5, 26, M) if M > 1 else 20)
    check(rounded(l, name), name, token, np.float32(np.full(M, dlp)).astype(np.float64), np.float32(np.full(M, dh)).astype(np.float64))


@pytest.mark.parametrize("dlp,dh", WEIGHTS)
def test_sure_tokens_of_far_rows(dlp, dh):
    """Logits so large that a row takes the differences; their steps are 2^-4."""
    r = np.random.default_rng(1)
    M, V = 100, 300
    l, token = np.round(r.normal(size=(M, V)) * 16) / 16, r.integers(0, V, M)
    l[np.arange(M), token] = np.round((np.log(V) + np.linspace(5, 26, M)) * 16) / 16
    l += 2.0 ** 20 - 64
    assert np.array_equal(l, rounded(l, "f32"))
    check(l, "f32", token, np.float32(np.full(M, dlp)).astype(np.float64), np.float32(np.full(M, dh)).astype(np.float64))


@pytest.mark.parametrize("name", ["f32", "bf16"])
def test_tokens_that_have_nothing(name):
    """The given token's share is 0, beside infinite, enormous and far logits, and some of the others: dlogprob is all it gets."""
    l = np.zeros((5, 40))
    l[0, 7] = l[0, 9] = np.inf
    l[1, 7], l[1, 3] = 3e38, -3e38
    l[2, 7], l[2, 3] = 400.0, -100.0
    l[3, 3] = -1e30
    l[4, 7], l[4, 3] = 2.0 ** 21, -2.0 ** 21
    token, dlp, dh = np.full(5, 3), np.full(5, 0.5), np.full(5, 2.0)
    got = score_gradient(rounded(l, name), name, token, dlp, dh)
    check_score_gradient(rounded(l, name), name, token, dlp, dh, got)
    assert (got[np.arange(5), token] == 0.5).all()
