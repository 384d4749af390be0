"""The operators' oracle against facts from elsewhere (no GPU): gradients against differences, e4m3 against the framework's
conversion, the draw against its definition by hand."""
import numpy as np
import pytest
import torch

from oracle import lm_ops as oracle


def test_recurrence_is_the_cell_with_gates_of_the_input_only():
    rng = np.random.default_rng(0)
    P = rng.standard_normal((4, 1, 8))
    h, c, before = oracle.scan_forward(P)
    s = 0.0
    for t in range(4):
        f, i, o, g = P[t, 0].reshape(4, 2)[:, 0]
        assert before[t, 0, 0] == pytest.approx(s)
        s = s / (1 + np.exp(-f)) + np.tanh(g) / (1 + np.exp(-i))
        assert h[t, 0, 0] == pytest.approx(np.tanh(s) / (1 + np.exp(-o)))
    assert c[0, 0] == pytest.approx(s)
    back = oracle.scan_forward(P[::-1], reverse=True)
    assert np.allclose(back[0][::-1], h) and np.allclose(back[1], c)


@pytest.mark.parametrize("reverse", [False, True])
def test_gradient_of_the_recurrence(reverse):
    rng = np.random.default_rng(1)
    T, Bn, H = 7, 3, 4
    P, c0, dh, dcT, n = rng.standard_normal((T, Bn, 4 * H)), rng.standard_normal((Bn, H)), rng.standard_normal((T, Bn, H)), rng.standard_normal((Bn, H)), [7, 0, 3]
    value = lambda P, c0: sum((a * b).sum() for a, b in zip(oracle.scan_forward(P, n, c0, reverse), (dh, dcT)))  # noqa: E731
    dP, dc0 = oracle.scan_backward(P, oracle.scan_forward(P, n, c0, reverse)[2], dh, dcT, n, reverse)
    for at in [(0, 0, 1), (2, 2, 5), (6, 0, 15), (3, 2, 0), (1, 1, 2)]:
        e = np.zeros_like(P)
        e[at] = 1e-6
        assert dP[at] == pytest.approx((value(P + e, c0) - value(P - e, c0)) / 2e-6, abs=1e-8)
    e = np.zeros_like(c0)
    e[1, 2] = 1e-6
    assert dc0[1, 2] == pytest.approx((value(P, c0 + e) - value(P, c0 - e)) / 2e-6, abs=1e-8)


def test_gradient_of_the_norm():
    rng = np.random.default_rng(2)
    s, w, dy = torch.tensor(rng.standard_normal((3, 10)), requires_grad=True), torch.tensor(rng.standard_normal(10), requires_grad=True), torch.tensor(rng.standard_normal((3, 10)))
    y = s * torch.rsqrt(s.square().mean(1, keepdim=True) + 1e-5) * w
    want, rstd = oracle.rmsnorm(s.detach().numpy(), w.detach().numpy(), 1e-5)
    assert np.allclose(want, y.detach().numpy(), rtol=1e-14)
    y.backward(dy)
    dx, dw = oracle.rmsnorm_backward(s.detach().numpy(), w.detach().numpy(), rstd, dy.numpy(), None)
    assert np.allclose(dx, s.grad.numpy(), rtol=1e-12, atol=1e-13) and np.allclose(dw, w.grad.numpy(), rtol=1e-12)


def test_e4m3_is_the_types_own_rounding():
    rng = np.random.default_rng(3)
    x = (rng.standard_normal(20000) * np.exp(rng.uniform(-9, 5, 20000))).clip(-448, 448).astype(np.float32)
    x = np.concatenate([x, np.float32(oracle._BETWEEN), -np.float32(oracle._BETWEEN), np.float32([0, -0.0, 448, -448, 2.0 ** -10, 1e-30])])
    want = torch.from_numpy(x).to(torch.float8_e4m3fn)
    assert np.array_equal(oracle.e4m3_encode(x), want.view(torch.uint8).numpy())
    assert np.array_equal(oracle.e4m3_decode(oracle.e4m3_encode(x)), want.double().numpy())
    codes, scale = oracle.quantize(np.full((2, 130), 3.0, np.float32))
    assert scale.shape == (2, 2) and (oracle.e4m3_decode(codes) == 448).all()
    assert np.allclose(oracle.matmul(codes, scale, codes, scale, 1)[0], 9 * 130)


def test_draw_by_hand():
    l = np.log([0.1, 0.4, 0.3, 0.2])
    assert [oracle.sample(l, u)[0] for u in (0.0, 0.09, 0.11, 0.49, 0.51, 0.81, 0.99)] == [0, 0, 1, 1, 2, 3, 3]
    assert oracle.sample(l, 0.3, top_k=2) == (1, pytest.approx(4 / 7), 2)
    assert oracle.sample(l, 0.3, top_p=0.41) == (1, pytest.approx(4 / 7), 2)
    assert oracle.sample(l, 0.3, top_p=0.39) == (1, pytest.approx(1.0), 1)
    assert oracle.sample(l, 0.999, min_p=0.6) == (2, pytest.approx(3 / 7), 2)
    assert oracle.sample(l, 0.999, temperature=0) == (1, 1.0, 1)
    assert oracle.sample(l, 0.5, allowed=[1, 0, 0, 1]) == (3, pytest.approx(2 / 3), 2)
    assert oracle.sample([-np.inf, np.nan], 0.5) == (-1, 0.0, 0)
    assert oracle.sample([2.0, 2.0, 2.0], 0.9, top_k=2)[0] == 1
