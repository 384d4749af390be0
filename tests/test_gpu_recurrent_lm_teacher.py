"""examples/recurrent_lm.py: its losses and their gradients by the logits, and a student of a teacher's words, end to end."""
import importlib.util
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lm():
    spec = importlib.util.spec_from_file_location("recurrent_lm_example", os.path.join(ROOT, "examples", "recurrent_lm.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_losses_and_their_gradients(lm):
    import torch
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    logits = torch.randn((30, 200), generator=gen, device="cuda") * 3
    token = torch.randint(0, 200, (30,), generator=gen, device="cuda", dtype=torch.int32)
    _, *teacher = lm.scores(torch.randn((30, 200), generator=gen, device="cuda") * 3, token, 16)
    x = logits.double().cpu().requires_grad_()
    log_p = torch.log_softmax(x, 1)
    first, t = teacher[0].cpu().long(), teacher[1].double().cpu().exp()
    rest = 1 - t.sum(1)
    s = log_p.exp()
    far = (t * (t.log() - log_p.gather(1, first))).sum(1) + rest * (rest.log() - (1 - s.gather(1, first).sum(1)).log())
    for (loss, grad), plain in ((lm.likelihood_loss(logits, token), -log_p.gather(1, token.cpu().long()[:, None]).mean()), (lm.teacher_loss(logits, teacher), far.mean())):
        want, = torch.autograd.grad(plain, x, retain_graph=True)
        # the mean of 30 fp32 numbers of up to 20; gradients up to 1 / 30, each from an exponential with 2^-24 of up to 20 times itself and a few roundings
        assert abs(float(loss) - float(plain.detach())) < 30 * 20 * 2.0 ** -24
        assert float((grad.double().cpu() - want).abs().max()) < (20 + 8) * 2.0 ** -24 / 30
        assert float(grad.sum(1).abs().max()) < 200 * (20 + 8) * 2.0 ** -24 / 30


def test_gradient_reaches_every_parameter(lm):
    import torch
    teacher_model, student = lm.RecurrentLm(150, 64, 1, seed=1), lm.RecurrentLm(150, 32, 2, seed=2)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(4)
    tokens = torch.randint(0, 150, (21, 3), generator=gen, device="cuda")
    _, *teacher = lm.scores(teacher_model.forward(tokens[:-1])[0], tokens[1:].reshape(-1).to(torch.int32), 20)
    loss, grad = student.gradient(tokens[:-1], tokens[1:], teacher)
    assert float(loss) > 0 and set(grad) == set(student.params)
    assert all(bool(g.isfinite().all()) and float(g.abs().max()) > 0 for g in grad.values())


def test_command():
    r = subprocess.run([sys.executable, os.path.join(ROOT, "examples", "recurrent_lm.py"), "--words", "120", "--units", "64", "--blocks", "1", "--prompt", "12",
                        "--generate", "4", "--train", "2", "--student", "32"], capture_output=True, text=True, timeout=110)
    assert r.returncode == 0, r.stderr[-2000:]
    assert "student: from the teacher" in r.stdout
