"""Distillation of rows without a teacher (a list of no words, as a padded row has it, and no teacher_lse): loss and gradient are 0, whatever the
student's row holds."""
import numpy as np
import pytest

from tests.lm_ops_util import rounded
from tests.test_gpu_scores import distill, teacher

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("M,V", [(8, 3000), (8, 70003), (600, 300)])
def test_no_loss_and_no_gradient(M, V, name):
    r = np.random.default_rng(4)
    l = r.normal(size=(M, V))
    words, z, _ = teacher(l, r, 5, 1.0, False)
    l[0], l[1], l[2, ::3], l[3], l[5, 7] = np.nan, -np.inf, np.inf, 1e30, np.nan
    words[:6] = -1
    words[2] = [V, -3, 1 << 30, V, -1]
    z[4] = np.nan
    loss, grad = distill(rounded(l, name), name, words, z, 1.0, None, np.ones(M))
    assert (loss[:6] == 0).all() and (grad[:6] == 0).all()
    assert np.isfinite(loss[6:]).all() and np.isfinite(grad[6:]).all() and (grad[6:] != 0).any(1).all()
    same, _ = distill(rounded(l, name), name, words, z, 1.0, None, np.ones(M), in_place=True)
    assert np.array_equal(same, loss)
