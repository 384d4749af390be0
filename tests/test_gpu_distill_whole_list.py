"""Distillation where the list is the whole vocabulary: there are no other words, and what rounding leaves of 1 is nobody's share."""
import importlib.util
import os
import subprocess
import sys

import numpy as np
import pytest

from oracle import lm_ops as O
from tests.lm_ops_util import U32, rounded
from tests.test_gpu_scores import check_distill, distill

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def lists(r, M, V, heat):
    z = np.float32(r.normal(size=(M, V)) * 3).astype(np.float64)
    words = r.permuted(np.tile(np.arange(V), (M, 1)), axis=1)
    lse = np.float32(np.log(np.exp(z / heat).sum(1))).astype(np.float64)
    return z, words, np.take_along_axis(z, words, 1), lse


def plain(l, z, heat, dloss):
    """The divergence over the whole vocabulary, and its gradient, from two softmaxes in 64 bits"""
    log_t, log_s = (x / heat - np.log(np.exp(x / heat).sum(1, keepdims=True)) for x in (z, l))
    loss = heat ** 2 * (np.exp(log_t) * (log_t - log_s)).sum(1)
    return loss, dloss[:, None] * heat * (np.exp(log_s) - np.exp(log_t))


@pytest.mark.parametrize("heat", [1.0, 2.0])
@pytest.mark.parametrize("V", [1, 2, 28, 200])
def test_oracle_has_no_share_for_nobody(V, heat):
    r = np.random.default_rng(V)
    z, words, listed, lse = lists(r, 50, V, heat)
    l, dloss = r.normal(size=(50, V)) * 3, r.normal(size=50)
    loss, grad = O.distill(l, words, listed, heat, lse, dloss)
    want, want_grad = plain(l, z, heat, dloss)
    # shares are off by what lse has been rounded by, up to 8 and so 2^-21; the logarithms they are multiplied with are up to 30
    assert np.abs(loss - want).max() < heat ** 2 * 2.0 ** -21 * 30 and np.abs(grad - want_grad).max() < 2.0 ** -21 * heat * np.abs(dloss).max()


def test_oracle_keeps_the_share_of_others():
    """One word outside the list, or one listed twice or not at all: its share counts as before."""
    l = np.log(np.array([[0.5, 0.3, 0.2]]))
    for words, z in (([0, 1], [0.6, 0.3]), ([0, 1, 1], [0.6, 0.3, 0.05]), ([0, 1, 3], [0.6, 0.3, 0.05])):
        loss, grad = O.distill(l, np.array([words]), np.log(np.array([z])), 1.0, np.zeros(1), np.ones(1))
        assert np.isclose(loss[0], 0.6 * np.log(0.6 / 0.5) + 0.1 * np.log(0.1 / 0.2)) and np.allclose(grad[0], [-0.1, 0, 0.1])


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("heat", [1.0, 2.0])
@pytest.mark.parametrize("V", [1, 2, 28, 200, 256])
def test_loss_is_the_divergence(V, heat, name):
    r = np.random.default_rng(V)
    z, words, listed, lse = lists(r, 60, V, heat)
    l, dloss = rounded(r.normal(size=(60, V)) * 3, name), np.float32(r.normal(size=60)).astype(np.float64)
    got = distill(l, name, words, listed, heat, lse, dloss)
    assert np.isfinite(got[0]).all()
    check_distill(l, name, words, listed, heat, lse, dloss, got)
    want, _ = plain(l, z, heat, dloss)
    # beside the loss's own rounding what lse has been rounded by, as above
    assert (np.abs(got[0] - want) < heat ** 2 * 2.0 ** -21 * 30 + 2 * U32 * np.abs(want)).all()
    near, _ = distill(rounded(z, name), name, words, listed, heat, lse, dloss)
    if name == "f32":           # the student is the teacher
        assert (np.abs(near) < heat ** 2 * 2.0 ** -21 * 30).all()


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["f32", "bf16"])
def test_lists_that_only_look_whole(name):
    """V words of which one is twice, or none: somebody is left, and the share is theirs."""
    r = np.random.default_rng(7)
    V = 40
    z, words, listed, lse = lists(r, 12, V, 1.0)
    words[::3, 5] = words[::3, 4]
    words[1::3, 5] = -1
    l, dloss = rounded(r.normal(size=(12, V)), name), np.float32(r.normal(size=12)).astype(np.float64)
    lse = np.float32(lse + 0.01).astype(np.float64)         # what the device gets
    check_distill(l, name, words, listed, 1.0, lse, dloss, distill(l, name, words, listed, 1.0, lse, dloss))


@pytest.mark.gpu
def test_student_of_a_small_vocabulary():
    """The example's teacher lists 32 words, here all there are."""
    import torch
    spec = importlib.util.spec_from_file_location("recurrent_lm_small", os.path.join(ROOT, "examples", "recurrent_lm.py"))
    lm = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(lm)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)
    logits = torch.randn((200, 28), generator=gen, device="cuda") * 3
    _, *teacher = lm.scores(logits, torch.zeros(200, dtype=torch.int32, device="cuda"), 28)
    loss, grad = lm.teacher_loss(logits, teacher)
    assert abs(float(loss)) < 2.0 ** -21 * 30 and float(grad.abs().max()) < 2.0 ** -20
    r = subprocess.run([sys.executable, os.path.join(ROOT, "examples", "recurrent_lm.py"), "--words", "20", "--units", "64", "--blocks", "1", "--prompt", "12",
                        "--generate", "4", "--train", "2", "--student", "32"], capture_output=True, text=True, timeout=110)
    assert r.returncode == 0, r.stderr[-2000:]
    line = [x for x in r.stdout.splitlines() if x.startswith("student: from the teacher")][0]
    assert "inf" not in line and "nan" not in line, line
