"""The draw of a token where a row stops fitting into the compute unit's memory, where the waves' runs end inside the row, and
where the border of a cold row's top_k lies far from its largest logit."""
import numpy as np
import pytest

from lm_ops_util import rounded
from test_gpu_sample import _check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("V,dtype", [(2048, "f32"), (2049, "f32"), (4096, "bf16"), (4097, "bf16"), (12289, "f32"), (28672, "f32"), (28673, "f32"),
                                     (57344, "bf16"), (57345, "bf16")])
def test_sizes_around_the_held_rows(V, dtype):
    rng = np.random.default_rng(V)
    M = 3
    logits = rounded(rng.standard_normal((M, V)) * 2.5, dtype)
    allowed = (rng.random((M, V)) < 0.8).astype(np.uint8)
    logits[allowed == 0] = np.nan
    u = np.array([0.0, np.float32(1 - 2.0 ** -24), 0.37], np.float32)
    _check(logits, u, dtype, allowed=allowed)
    _check(logits, u, dtype, allowed=allowed, top_k=40, top_p=0.9, pad=1, off=1)
    _check(logits, u, dtype, allowed=allowed, top_p=0.97, min_p=0.001)


@pytest.mark.parametrize("V", [1000, 5000])
def test_cold_rows(V):
    """Low temperatures: what top_k still keeps weighs next to nothing."""
    rng = np.random.default_rng(V)
    M = 6
    logits = rounded(rng.standard_normal((M, V)) * np.array([2.5, 2.5, 20.0, 200.0, 1e30, 0.01])[:, None], "f32")
    k = np.array([V - 3, V // 2, V - 1, V // 3, V // 2, V - 7])
    _check(logits, rng.random(M), top_k=k, temperature=0.05)
    _check(logits, rng.random(M), top_k=k, top_p=0.9, temperature=0.3)


def test_one_launch_after_another_in_both_directions_of_filters():
    """Rows with and without each filter side by side: steps that one row takes and its neighbour does not."""
    rng = np.random.default_rng(9)
    M, V = 40, 3000
    logits = rounded(rng.standard_normal((M, V)) * 2.5, "f32")
    logits[::7] = np.round(logits[::7])                      # many equal ones
    logits[3] = -np.inf
    _check(logits, rng.random(M), top_k=rng.choice([0, 1, 7, 600, 2999], M), top_p=rng.choice([1.0, 0.0, 0.5, 0.99], M),
           min_p=rng.choice([0.0, 0.02, 1.0], M), temperature=rng.choice([0.0, 0.2, 1.0, 3.0], M))
