"""Distillation of a student whose words outside the list are all minus infinity: they get no gradient, whatever the teacher leaves them.  What
it leaves is a share that nobody has (an infinite loss), or no more than the rounding of the teacher's numbers (no share)."""
import numpy as np
import pytest

from oracle import lm_ops as O
from tests.lm_ops_util import rounded
from tests.test_gpu_scores import check_distill, distill, teacher


def student(seed, M, V, K, name="f32"):
    """Rows whose listed words alone exist; the last one whole"""
    r = np.random.default_rng(seed)
    l = r.normal(size=(M, V)) * 2
    words, z, _ = teacher(l, r, K, 1.0, False)
    masked = np.full((M, V), -np.inf)
    np.put_along_axis(masked, words, np.take_along_axis(l, words, 1), 1)
    masked[-1] = l[-1]
    return rounded(masked, name), words, z, r


def own_lse(z, heat=1.0):
    """log of the list's own sum, in fp32: a teacher that is masked as the student is"""
    return np.float32(np.log(np.exp(z / heat).sum(1))).astype(np.float64)


def test_oracle():
    l = np.array([[0.0, 0.0, -np.inf, -np.inf]])
    loss, grad = O.distill(l, np.array([[0, 1]]), np.log(np.array([[0.5, 0.2]])), 1.0, np.zeros(1), np.ones(1))
    assert loss[0] == np.inf and np.allclose(grad, [[0, 0.3, 0, 0]])


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("M,V,K", [(9, 50, 6), (5, 9000, 40), (600, 700, 3), (3, 70003, 64)])
def test_nobody_has_the_share(M, V, K, name):
    l, words, z, r = student(2, M, V, K, name)
    dloss = np.float32(r.normal(size=M)).astype(np.float64)
    for off in (0.5, 1e-4, -0.1):
        lse = np.float32(own_lse(z) + off).astype(np.float64)
        got = distill(l, name, words, z, 1.0, lse, dloss)
        check_distill(l, name, words, z, 1.0, lse, dloss, got)
        assert (got[1][:-1][l[:-1] == -np.inf] == 0).all()
        assert (np.isposinf(got[0][:-1]) == (off > 0)).all() and np.isfinite(got[0][-1])


def test_oracle_takes_rounding_for_no_share():
    l, words, z, r = student(1, 200, 50, 6)
    loss, grad = O.distill(l, words, z, 1.0, own_lse(z), np.ones(200))
    assert np.isfinite(loss).all() and (grad[:-1][l[:-1] == -np.inf] == 0).all()
    loss, _ = O.distill(l, words, z, 1.0, own_lse(z) + 1e-5, np.ones(200))     # more than rounding
    assert (loss[:-1] == np.inf).all() and np.isfinite(loss[-1])


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("heat", [1.0, 0.5, 3.0])
def test_rounding_is_no_share(heat, name):
    l, words, z, r = student(3, 300, 50, 6, name)
    dloss = np.float32(r.normal(size=300)).astype(np.float64)
    lse = own_lse(z, heat)
    got = distill(l, name, words, z, heat, lse, dloss)
    assert np.isfinite(got[0]).all() and np.isfinite(got[1]).all()
    rows = slice(0, 299)        # the last one has others, whose share is as good as its rounding
    check_distill(l[rows], name, words[rows], z[rows], heat, lse[rows], dloss[rows], (got[0][rows], got[1][rows]))
