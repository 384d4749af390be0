"""The unit in which the weights of a draw are counted, as the header states it, and settings that are NaN."""
import math

import numpy as np
import pytest

from lm_ops_util import dev, ptr, workspace
from paper_1901_10997_amd import binding as B

pytestmark = pytest.mark.gpu


def _draw(logits, u, top_p=None, min_p=None):
    import torch
    M, V = logits.shape
    ld, ud = dev(np.float32(logits)), dev(np.float32(u))
    row = lambda v: None if v is None else torch.full((M,), v, device="cuda:0")  # noqa: E731
    p, m = row(top_p), row(min_p)
    token, kept = torch.empty(M, dtype=torch.int32, device="cuda:0"), torch.empty(M, dtype=torch.int32, device="cuda:0")
    prob = torch.empty(M, device="cuda:0")
    ws = workspace(B.lstm_sample_workspace_bytes(M, V))
    B.lstm_sample(M, V, B.LSTM_F32, ptr(ld), V, None, 0, None, None, ptr(p), ptr(m), ptr(ud), ptr(token), ptr(prob), ptr(kept), ptr(ws), ws.numel())
    torch.cuda.synchronize()
    return token.cpu().numpy(), prob.cpu().numpy(), kept.cpu().numpy()


@pytest.mark.parametrize("V", [2, 3, 256, 1024, 1025, 2048, 2049, 4096, 4097, 30000, 131072, 1 << 20])
def test_unit_of_the_weights(V):
    S = min(51, 62 - math.ceil(math.log2(V)))
    # one token of weight 1, half of the others a quarter of a unit below half a unit, the rest above it
    logits = np.full((1, V), -(S + 1 + 0.41) * math.log(2))             # 0.75 of half a unit
    over = np.arange(1, V)[::2]
    logits[0, over] = -(S + 1 - 0.32) * math.log(2)                     # 1.25 of half a unit
    logits[0, 0] = 0
    for min_p, stay in ((None, V), (0.0, V), (1e-30, 1 + len(over)), (2.0 ** -S, 1 + len(over)), (1.5 * 2.0 ** -S, 1)):
        token, prob, kept = _draw(logits, [0.0], min_p=min_p)
        assert (token[0], kept[0]) == (0, stay), (V, min_p, kept)
        assert prob[0] == np.float32(1 / (1 + (len(over) if stay > 1 else 0) * 2.0 ** -S))


def test_settings_that_are_nan():
    rng = np.random.default_rng(4)
    logits = rng.standard_normal((5, 300))
    logits[:, 17] = logits[:, 200] = 5
    nan = float("nan")
    assert (_draw(logits, np.full(5, 0.5), top_p=nan)[2] == 300).all()
    assert (_draw(logits, np.full(5, 0.5), min_p=nan)[2] == 2).all()
    for a, b in zip(_draw(logits, np.full(5, nan)), _draw(logits, np.zeros(5))):
        assert np.array_equal(a, b)
