"""The temperature of a distillation is taken as it is given, in 64 bits: teacher_lse is the caller's, of that temperature, and where the list has nearly all
mass the share of the others is a difference that the temperature's rounding to fp32 would be all of.

Tolerance: what check_distill grants, at the exact temperature."""
import ctypes

import numpy as np
import pytest

from oracle import lm_ops as O
from paper_1901_10997_amd import binding as B
from tests import test_gpu_scores as S
from tests.lm_ops_util import HALF, U32, close, rounded


def test_entries_take_64_bits():
    lib = B.load()
    for name in ("lstm_distill_forward", "lstm_distill_backward"):
        assert getattr(lib, name).argtypes[11] is ctypes.c_double


def case(seed, M, V, K, heat, name):
    """A teacher whose list leaves the others a share of 1e-7 to 1e-2, and the lse in 64 bits rounded once"""
    r = np.random.default_rng(seed)
    z = np.float32(r.normal(size=(M, V))).astype(np.float64)
    words = np.argsort(-z, axis=1)[:, :K]
    lift = np.float32(heat * r.uniform(np.log(V / 1e-2), np.log(V / 1e-7), (M, 1)))
    np.put_along_axis(z, words, np.float32(np.take_along_axis(z, words, 1) + lift).astype(np.float64), 1)
    lse = np.float32(np.log(np.exp((z - 20 * heat) / heat).sum(1)) + 20).astype(np.float64)
    l = rounded(z + r.normal(size=z.shape) * 0.3, name)
    return l, words, np.take_along_axis(z, words, 1), lse, np.float32(r.normal(size=M)).astype(np.float64)


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("heat", [0.53, 1.7, 3.3, 2.0])
@pytest.mark.parametrize("M,V,K", [(40, 500, 8), (7, 20003, 64), (600, 2500, 3)])
def test_distill(M, V, K, heat, name):
    l, words, z, lse, dloss = case(M, M, V, K, heat, name)
    got = S.distill(l, name, words, z, heat, lse, dloss)
    loss, grad = O.distill(l, words, z, heat, lse, dloss)
    log_s = l / heat - l.max(1, keepdims=True) / heat
    log_s -= np.log(np.exp(log_s).sum(1, keepdims=True))
    s = np.exp(log_s)
    mean = (s * abs(log_s)).sum(1)
    outside = np.ones(l.shape, bool)
    np.put_along_axis(outside, words, False, 1)
    s_r = (s * outside).sum(1)
    far = np.take_along_axis(abs(log_s), words, 1).max(1) + abs(np.log(s_r)) + 1 + mean
    close(got[0], loss, heat ** 2 * U32 * (2 * far + 12) + U32 * abs(loss), "loss")
    w = abs(dloss[:, None]) * heat
    want = s - grad / (dloss[:, None] * heat)
    # dloss heat, one product in fp32, besides
    tol = U32 * w * (s + abs(want)) * (abs(log_s) + mean[:, None] + 16) + 2 * w * 2.0 ** -126
    close(got[1], grad, tol + (HALF[name] + U32) * abs(grad), "dlogits")
