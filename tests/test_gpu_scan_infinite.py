"""Gated linear recurrence and its gradient with infinite and NaN states, pre-activations and gradients, where gates are so small
that their product over a few steps is below the smallest number: as step by step, however time is cut."""
import numpy as np
import pytest

from lm_ops_util import HALF, U32, close, rounded
from oracle import lm_ops as oracle
from test_gpu_scan import _run

pytestmark = pytest.mark.gpu

# one run, some tiles in one piece, some with few workgroups (time is cut), enough workgroups that it is not
SIZES = [(7, 2, 66), (33, 2, 66), (64, 1, 70), (130, 1, 66), (700, 2, 130), (300, 20, 1000)]


def _inputs(T, Bn, H, dtype, seed):
    rng = np.random.default_rng(seed)
    P = rng.standard_normal((T, Bn, 4 * H))
    P[:, :, :H] -= rng.choice([0.0, 6.0, 20.0, 60.0], H)        # 60: 2^-86
    return rng, rounded(P, dtype), rounded(rng.standard_normal((T, Bn, H)), dtype), rng.standard_normal((Bn, H)).astype(np.float32), rng.standard_normal((Bn, H)).astype(np.float32)


def _same(got, want, tol, what):
    """close(), and infinities of the same sign."""
    close(got, want, tol, what)
    far = np.isinf(want)
    assert np.array_equal(got[far], want[far]), what


@pytest.mark.parametrize("T,Bn,H", SIZES)
@pytest.mark.parametrize("dtype,reverse", [("f32", False), ("bf16", True)])
def test_infinite_first_state(T, Bn, H, dtype, reverse):
    rng, P, dh, c0, dcT = _inputs(T, Bn, H, dtype, T)
    c0[0, :20], c0[-1, 30:40], c0[0, 41:44] = np.inf, -np.inf, np.nan
    place = T // 2
    P[place, 0, 10:14] = -np.inf                            # a forget gate of zero: 0 * infinity
    lengths = None if Bn == 1 else rng.integers(T // 2 + 1, T + 1, Bn).astype(np.int32)
    bh, cT, states, *_ = _run(T, Bn, H, dtype, reverse, "tb", 0, 0, P, dh, c0, dcT, lengths, train=False)
    with np.errstate(invalid="ignore"):
        h, c, _ = oracle.scan_forward(P, lengths, c0, reverse)
    assert np.isinf(c[0, :10]).all() and np.isnan(c[0, 10:14]).all() and np.isnan(c[0, 41:44]).all()
    # gates to 16 halves of a step each, on states of at most a few units' size
    tol = 48 * U32 * 8 * (1 + np.abs(c0[np.isfinite(c0)]).max())
    _same(bh.get(), h, tol + HALF[dtype] * np.abs(np.nan_to_num(h)), "h")
    _same(cT.get(), c, tol, "cT")


@pytest.mark.parametrize("T,Bn,H", SIZES)
@pytest.mark.parametrize("dtype,reverse", [("f32", False), ("bf16", True)])
def test_infinite_gradients(T, Bn, H, dtype, reverse):
    """Of the final state, and of h in the middle: everything in front of them is infinite, what is behind them is not."""
    rng, P, dh, c0, dcT = _inputs(T, Bn, H, dtype, T + 1)
    dcT[0, :20], dcT[-1, 30:40], dcT[0, 41:44] = np.inf, -np.inf, np.nan
    dh[T // 2, 0, 50:56] = np.inf
    P, dh = rounded(P, dtype), rounded(dh, dtype)
    c0 = np.where(np.abs(c0) < 0.1, 0.5, c0).astype(np.float32)
    lengths = None if Bn == 1 else rng.integers(T // 2 + 1, T + 1, Bn).astype(np.int32)
    bh, cT, states, bdp, dc0 = _run(T, Bn, H, dtype, reverse, "tb", 0, 0, P, dh, c0, dcT, lengths)
    _, _, before = oracle.scan_forward(P, lengths, c0, reverse)
    with np.errstate(invalid="ignore"):
        dP, d0 = oracle.scan_backward(P, before, dh, dcT, lengths, reverse)
    assert np.isinf(d0[0, :20]).all() and np.isnan(d0[0, 41:44]).all() and np.isinf(d0[0, 50:56]).all() and np.isfinite(d0[0, 56:]).all()
    big = max(1.0, np.abs(dP[np.isfinite(dP)]).max())
    tol = 2 * 48 * U32 * 8 * (1 + np.abs(c0).max()) * big
    _same(dc0.get(), d0, tol, "dc0")
    got, H_ = bdp.get(), H
    finite = np.isfinite(dP)
    assert np.array_equal(finite, np.isfinite(got))
    assert (np.abs(got - dP)[finite] <= tol + HALF[dtype] * np.abs(dP[finite])).all()


@pytest.mark.parametrize("T,Bn,H", [(700, 2, 130), (300, 20, 1000)])
def test_nan_and_infinite_gates_across_the_pieces_of_time(T, Bn, H):
    """A NaN reaches every later step of its unit and nothing else; a forget gate at minus infinity lets nothing through, at plus
    infinity everything, wherever time is cut."""
    rng, P, dh, c0, dcT = _inputs(T, Bn, H, "f32", 3)
    P[:, :, :H] = rng.choice([np.inf, 40.0, 3e38], (T, Bn, H))
    P[T // 3, :, :H:3] = -np.inf
    P[T // 2, 0, 5], P[T // 4, 1, 2 * H + 9], P[5, 0, 3 * H + 12] = np.nan, np.nan, np.nan
    P[:, :, H:2 * H] -= 8                                   # states stay small although nothing is forgotten
    bh, cT, *_ = _run(T, Bn, H, "f32", False, "tb", 0, 0, P, dh, c0, None, None, train=False)
    h, c, _ = oracle.scan_forward(P, None, c0)
    assert np.isnan(h).sum() == (T - T // 2) + 1 + (T - 5)
    tol = 48 * U32 * T * (1 + np.abs(c0).max())
    close(bh.get(), h, tol)
    close(cT.get(), c, tol)
    assert (np.abs(c[0, 0] - c0[0, 0]) < np.abs(c0[0, 0]) + 10)


@pytest.mark.parametrize("T,Bn,H,dtype", [(1, 3, 70, "f32"), (40, 3, 70, "bf16"), (700, 3, 70, "f32")])
@pytest.mark.parametrize("reverse", [False, True])
def test_lengths_below_zero_and_above_the_steps(T, Bn, H, dtype, reverse):
    """They are taken as 0 and as all steps."""
    _, P, dh, c0, dcT = _inputs(T, Bn, H, dtype, 9)
    some = [_run(T, Bn, H, dtype, reverse, "tb", 0, 0, P, dh, c0, dcT, np.array(n, np.int32)) for n in
            ([-5, T + 7, -2 ** 31], [0, T, 0], [2 ** 31 - 1, -1, T], [T, 0, T])]
    for a, b in ((0, 1), (2, 3)):
        for i in (0, 1, 3, 4):
            assert np.array_equal(some[a][i].get(), some[b][i].get())
    h, c, _ = oracle.scan_forward(P, [0, T, 0], c0, reverse)
    assert np.array_equal(some[0][1].get()[0], c0[0]) and not some[0][0].get()[:, 0].any()
    close(some[0][1].get(), c, 48 * U32 * 8 * (1 + np.abs(c0).max()))
