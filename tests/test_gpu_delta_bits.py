"""Gated delta rule with results in bf16, where what a result is summed from is far larger than the result: the products have all bits of fp32, and
the rounding to bf16 is that of the result alone.

Tolerance.  A result is a sum of products whose factors are fp32 values; the three planes of a factor hold its 24 bits, and of the planes'
products those below 2^-24 are left out.  Here at most two terms of a sum are not 0, each of six products of planes, and a term goes
through the update, the product and the join with what comes from the other steps: no more than 24 additions and
roundings, each off by half a step u of fp32 of the sum of the terms' magnitudes, and half a step of bf16 of the result.  (A factor cut to 16 bits is off by up to 128 u.)"""
import numpy as np
import pytest

from tests import delta_util as D
from tests.lm_ops_util import HALF, U32, close, rounded

pytestmark = pytest.mark.gpu
NEAR = 1 + 2.0 ** -12
MANY = [1, 64]          # sequences: one tile of columns to a workgroup, and two


def case(T, batch, heads, Dk, Dv):
    c = D.make(21, T, batch, heads, heads, Dk, Dv, "bf16", decay=None)
    for key in ("q", "k", "v", "beta", "S0", "dO", "dST"):
        c[key] = np.zeros_like(c[key])
    c["scale"] = 1.0
    return c


def fp32(x):
    return np.float32(x).astype(np.float64)


@pytest.mark.parametrize("batch", MANY)
def test_read_of_a_state(batch):
    """o = S0[0] + S0[1], two rows that are nearly each other's opposite; nothing is ever written."""
    c = case(70, batch, 8, 2, 20)
    r = np.random.default_rng(1)
    c["q"][:] = 1
    c["S0"][:, :, 0] = fp32(r.uniform(1, 2, c["S0"][:, :, 0].shape))
    c["S0"][:, :, 1] = fp32(-c["S0"][:, :, 0] * NEAR)
    o, _, _ = D.forward(c, D.buffers(c))
    want = np.broadcast_to(c["S0"].sum(2).reshape(1, batch, -1), c["v"].shape)
    size = np.broadcast_to(abs(c["S0"]).sum(2).reshape(1, batch, -1), c["v"].shape)
    close(o.get(), want, 24 * U32 * size + HALF["bf16"] * abs(want), "o")


@pytest.mark.parametrize("batch", MANY)
def test_read_of_a_block_s_own_updates(batch):
    """Two values written under two keys, read as their difference in the same block and in the next."""
    c = case(70, batch, 8, 2, 20)
    r = np.random.default_rng(2)
    k, q = c["k"].reshape(70, batch, 8, 2), c["q"].reshape(70, batch, 8, 2)
    k[0, ..., 0] = k[1, ..., 1] = 1
    q[2:, ..., 0], q[2:, ..., 1] = 1, -1
    c["v"][:2] = rounded(r.uniform(1, 2, (1, *c["v"].shape[1:])), "bf16")
    c["beta"][0] = fp32(r.uniform(0.2, 0.9, (batch, 8)))
    c["beta"][1] = fp32(c["beta"][0] * NEAR)
    o, _, _ = D.forward(c, D.buffers(c))
    v = c["v"][0].reshape(batch, 8, 20)
    want = np.zeros((70, batch, 160))
    want[2:] = ((c["beta"][0] - c["beta"][1])[..., None] * v).reshape(batch, 160)
    size = ((c["beta"][0] + c["beta"][1])[..., None] * v).reshape(batch, 160)
    close(o.get(), want, 24 * U32 * size + HALF["bf16"] * abs(want), "o")


def sizes(c, keep):
    """What the terms of dq and dk [T, batch, heads, Dk] come to in magnitude: the recurrence and its gradient with every sign plus.  `keep`: |1 - beta|, what a
    key's own row of the state keeps, in the place of 1 + beta."""
    T, batch, H = c["beta"].shape
    k, q = (abs(c[n].reshape(T, batch, H, -1)) for n in "kq")
    dO, b = abs(c["dO"].reshape(T, batch, H, -1)), c["beta"]
    S, front, d = abs(c["S0"]), [], abs(c["dST"])
    dq, dk = np.zeros(q.shape), np.zeros(k.shape)
    for t in range(T):
        front.append(S)
        S = S + np.einsum("bhd,bh,bhv->bhdv", k[t], keep(b[t]) - 1, np.einsum("bhd,bhdv->bhv", k[t], S))
        dq[t] = np.einsum("bhdv,bhv->bhd", S, dO[t])
    for t in range(T - 1, -1, -1):
        d = d + np.einsum("bhd,bhv->bhdv", q[t], dO[t])
        found, du = np.einsum("bhd,bhdv->bhv", k[t], front[t]), np.einsum("bhd,bhdv->bhv", k[t], d)
        dk[t] = np.einsum("bhdv,bh,bhv->bhd", d, b[t], found) + np.einsum("bh,bhdv,bhv->bhd", b[t], front[t], du)
        d = d + np.einsum("bhd,bh,bhv->bhdv", k[t], keep(b[t]) - 1, du)
    return dq.reshape(T, batch, -1), dk.reshape(T, batch, -1)


def check_gradient(c):
    s = D.buffers(c)
    _, _, kept = D.forward(c, s, states=True)
    out, _ = D.backward(c, s, kept)
    _, _, front = D.oracle_forward(c)
    want = D.O.delta_backward(*D.oracle_args(c), front, c["dO"], None, c["dST"])
    for name, w, size in zip(("dq", "dk"), want, sizes(c, lambda b: abs(1 - b))):
        close(out[name].get(), w, 24 * U32 * size + HALF["bf16"] * abs(w), name)


@pytest.mark.parametrize("batch", MANY)
def test_gradients_by_rows_that_cancel(batch):
    """Two columns of S0 that are nearly equal against gradients of opposite sign, a key of its own at every step."""
    c = case(12, batch, 8, 16, 2)
    r = np.random.default_rng(3)
    k, q = c["k"].reshape(12, batch, 8, 16), c["q"].reshape(12, batch, 8, 16)
    at = np.arange(12)
    k[at, ..., at] = 1
    q[at, ..., at] = 1
    c["beta"][:] = fp32(r.uniform(0.2, 0.9, c["beta"].shape))
    c["S0"][..., 0] = fp32(r.uniform(1, 2, c["S0"][..., 0].shape))
    c["S0"][..., 1] = fp32(c["S0"][..., 0] * NEAR)
    c["dST"][..., 0] = fp32(r.uniform(1, 2, c["dST"][..., 0].shape))
    c["dST"][..., 1] = -c["dST"][..., 0]
    dO = c["dO"].reshape(12, batch, 8, 2)
    dO[..., 0] = rounded(r.uniform(1, 2, dO[..., 0].shape), "bf16")
    dO[..., 1] = -dO[..., 0]
    check_gradient(c)


@pytest.mark.parametrize("batch", MANY)
def test_gradients_by_steps_that_cancel(batch):
    """A key's gradient through two later reads in the same block that are nearly each other's opposite."""
    c = case(12, batch, 8, 16, 2)
    r = np.random.default_rng(4)
    k, q = c["k"].reshape(12, batch, 8, 16), c["q"].reshape(12, batch, 8, 16)
    at = np.arange(8)
    k[at, ..., at + 1] = 1
    q[8, ..., 0], q[9, ..., 0] = 1, -1
    c["beta"][:8] = fp32(r.uniform(0.2, 0.9, c["beta"][:8].shape))
    c["S0"][:, :, 1:, 0] = fp32(-r.uniform(1, 2, c["S0"][:, :, 1:, 0].shape))
    c["S0"][:, :, 1:, 1] = fp32(c["S0"][:, :, 1:, 0] * NEAR)
    dO = c["dO"].reshape(12, batch, 8, 2)
    dO[8] = 1
    dO[9] = 1 + 2.0 ** -7, 1 - 2.0 ** -7
    check_gradient(c)
