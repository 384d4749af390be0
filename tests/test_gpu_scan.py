"""Gated linear recurrence and its gradient against the fp64 oracle: widths off every tile, one to many steps, segments cut
over workgroups, ragged lengths with empty sequences, both directions, layouts and alignments, junk where nothing may be read."""
import numpy as np
import pytest

from lm_ops_util import Buf, DTYPE, HALF, U32, close, dev, ptr, rounded, workspace
from oracle import lm_ops as oracle
from paper_1901_10997_amd import binding as B

pytestmark = pytest.mark.gpu

CASES = [
    # T, batch, H, dtype, reverse, ragged, layout ("tb": steps outermost, "bt": sequences outermost), pad, offset
    (1, 1, 1, "f32", False, False, "tb", 0, 0),
    (1, 3, 65, "bf16", False, True, "tb", 0, 0),
    (2, 1, 64, "f32", False, False, "tb", 0, 0),
    (15, 2, 63, "bf16", True, False, "tb", 0, 0),
    (16, 2, 66, "bf16", False, False, "bt", 0, 0),
    (17, 1, 130, "f32", True, False, "tb", 5, 3),
    (64, 3, 100, "bf16", False, True, "tb", 0, 0),
    (65, 2, 131, "bf16", True, True, "bt", 1, 1),
    (130, 5, 70, "f32", False, True, "bt", 2, 1),
    (127, 4, 256, "bf16", False, False, "tb", 8, 2),
    (300, 2, 96, "f32", True, True, "tb", 0, 0),
    (1000, 1, 34, "bf16", False, False, "tb", 0, 0),
    (1500, 1, 72, "f32", False, False, "tb", 0, 0),
    (1290, 2, 129, "bf16", True, True, "tb", 0, 0),
]


def _inputs(T, Bn, H, dtype, ragged, seed):
    rng = np.random.default_rng(seed)
    P = rng.standard_normal((T, Bn, 4 * H))
    P[:, :, :H] += rng.uniform(0, 4, H)                      # forget gates of short to long memory
    P = rounded(P, dtype)
    dh = rounded(rng.standard_normal((T, Bn, H)), dtype)
    c0, dcT = rng.standard_normal((Bn, H)).astype(np.float32), rng.standard_normal((Bn, H)).astype(np.float32)
    lengths = None
    if ragged:
        lengths = rng.integers(0, T + 1, Bn).astype(np.int32)
        lengths[0] = 0
        if Bn > 1:
            lengths[-1] = T
        for b in range(Bn):
            P[lengths[b]:, b] = np.nan                       # never read into a result
            dh[lengths[b]:, b] = np.nan
    return P, dh, c0, dcT, lengths


def _memory(P, H, lengths, reverse):
    """Largest sum of products of forget gates: how many steps' roundings a state carries."""
    T, Bn = P.shape[:2]
    f = oracle.sigmoid(P[:, :, :H])
    best = 1.0
    for b in range(Bn):
        n = T if lengths is None else int(lengths[b])
        m = np.zeros(H)
        for s in range(n):
            m = 1 + f[n - 1 - s if reverse else s, b] * m
            best = max(best, float(m.max()))
    return best


def _run(T, Bn, H, dtype, reverse, layout, pad, off, P, dh, c0, dcT, lengths, stream=None, train=True):
    order = [0, 1] if layout == "tb" else [1, 0]
    bp = Buf((T, Bn, 4 * H), dtype, pad, off, P, order)
    bh = Buf((T, Bn, H), dtype, pad, off, None, order)
    bdh = Buf((T, Bn, H), dtype, pad, off, dh, order)
    bdp = Buf((T, Bn, 4 * H), dtype, pad, off, None, order)
    states = Buf((-(-T // B.LSTM_SCAN_STEPS), Bn, H))
    cT, dc0 = Buf((Bn, H)), Buf((Bn, H))
    ln, c0d, dcd = dev(lengths), dev(c0), dev(dcT)
    ws = workspace(B.lstm_scan_workspace_bytes(T, Bn, H))
    B.lstm_scan_forward(T, Bn, H, DTYPE[dtype], int(reverse), bp.ptr, *bp.strides, ptr(ln), ptr(c0d), bh.ptr, *bh.strides, cT.ptr,
                        states.ptr if train else None, ws.data_ptr(), ws.numel(), stream)
    if train:
        ws.fill_(0x5A)
        B.lstm_scan_backward(T, Bn, H, DTYPE[dtype], int(reverse), bp.ptr, *bp.strides, ptr(ln), states.ptr, bdh.ptr, *bdh.strides,
                             ptr(dcd), bdp.ptr, *bdp.strides, dc0.ptr, ws.data_ptr(), ws.numel(), stream)
    return bh, cT, states, bdp, dc0


@pytest.mark.parametrize("T,Bn,H,dtype,reverse,ragged,layout,pad,off", CASES)
@pytest.mark.parametrize("state", [True, False])
def test_forward_and_gradient(T, Bn, H, dtype, reverse, ragged, layout, pad, off, state):
    P, dh, c0, dcT, lengths = _inputs(T, Bn, H, dtype, ragged, 7 * T + H)
    if not state:
        c0 = dcT = None
    bh, cT, states, bdp, dc0 = _run(T, Bn, H, dtype, reverse, layout, pad, off, P, dh, c0, dcT, lengths)
    h, c, before = oracle.scan_forward(P, lengths, c0, reverse)
    dP, d0 = oracle.scan_backward(P, before, dh, dcT, lengths, reverse)
    # a step rounds a handful of times: each gate to within 16 halves of a step (its argument's, the exponential's and the
    # reciprocal's), the products one each; a state carries the roundings of as many steps as its gates remember
    tol = 48 * U32 * _memory(np.nan_to_num(P), H, lengths, reverse)
    size = 1.0 + (0 if c0 is None else np.abs(c0).max())
    close(bh.get(), h, tol * size + HALF[dtype] * np.abs(h), "h")
    close(cT.get(), c, tol * size, "cT")
    close(states.get(), before[::B.LSTM_SCAN_STEPS], tol * size, "states")
    # the gradient runs through the same gates once more, on states that carry the forward's error; its largest values set
    # the size of what the roundings are relative to
    big = max(1.0, np.abs(dP).max(), np.abs(d0).max())
    close(bdp.get(), dP, 2 * tol * size * big + HALF[dtype] * np.abs(dP), "dP")
    close(dc0.get(), d0, 2 * tol * size * big, "dc0")


def test_gradient_against_differences():
    """The sum of h and cT with random weights, moved along random directions of P and c0."""
    T, Bn, H = 40, 2, 24
    P, dh, c0, dcT, _ = _inputs(T, Bn, H, "f32", False, 5)
    rng = np.random.default_rng(6)
    _, _, _, bdp, dc0 = _run(T, Bn, H, "f32", False, "tb", 0, 0, P, dh, c0, dcT, None)
    gP, g0 = bdp.get(), dc0.get()

    def value(P, c0):
        h, c, _ = oracle.scan_forward(P, None, c0)
        return (h * dh).sum() + (c * dcT).sum()

    for _ in range(3):
        vP, v0, step = rng.standard_normal(P.shape), rng.standard_normal(c0.shape), 1e-5
        want = (value(P + step * vP, c0 + step * v0) - value(P - step * vP, c0 - step * v0)) / (2 * step)
        got = (gP * vP).sum() + (g0 * v0).sum()
        # the central difference is off by its third derivative, about step^2, and the gradient by fp32 roundings
        assert abs(got - want) <= 1e-4 * np.sqrt((gP ** 2).sum() + (g0 ** 2).sum())


def test_pieces_give_the_whole():
    """A sequence read in pieces, single steps among them, with the state carried in place, is the sequence read at once."""
    T, Bn, H = 150, 3, 80
    P, dh, c0, _, _ = _inputs(T, Bn, H, "f32", False, 8)
    bh, cT, *_ = _run(T, Bn, H, "f32", False, "tb", 0, 0, P, dh, c0, None, None)
    import torch
    Pd, c = dev(P.astype(np.float32)), dev(c0)
    h = torch.empty((T, Bn, H), device="cuda:0")
    at = 0
    for n in (1, 1, 16, 1, 63, 64, 1, 3):
        ws = workspace(B.lstm_scan_workspace_bytes(n, Bn, H))
        B.lstm_scan_forward(n, Bn, H, B.LSTM_F32, 0, Pd[at].data_ptr(), Bn * 4 * H, 4 * H, None, c.data_ptr(), h[at].data_ptr(), Bn * H, H,
                            c.data_ptr(), None, ws.data_ptr(), ws.numel())
        at += n
    assert at == T
    tol = 48 * U32 * _memory(P, H, None, False) * (1 + np.abs(c0).max())
    close(h.double().cpu().numpy(), bh.get(), 2 * tol)
    close(c.double().cpu().numpy(), cT.get(), 2 * tol)


def test_no_steps_and_no_sequences():
    import torch
    c0 = torch.randn((3, 70), device="cuda:0")
    cT = torch.full((3, 70), 9.0, device="cuda:0")
    ws = workspace(B.lstm_scan_workspace_bytes(0, 3, 70))
    B.lstm_scan_forward(0, 3, 70, B.LSTM_F32, 0, None, 0, 0, None, c0.data_ptr(), None, 0, 0, cT.data_ptr(), None, ws.data_ptr(), ws.numel())
    torch.cuda.synchronize()
    assert torch.equal(c0, cT)
    B.lstm_scan_forward(0, 3, 70, B.LSTM_F32, 0, None, 0, 0, None, None, None, 0, 0, cT.data_ptr(), None, ws.data_ptr(), ws.numel())
    B.lstm_scan_backward(0, 3, 70, B.LSTM_F32, 0, None, 0, 0, None, None, None, 0, 0, c0.data_ptr(), None, 0, 0, c0.data_ptr(), ws.data_ptr(), ws.numel())
    B.lstm_scan_forward(4, 0, 70, B.LSTM_F32, 0, None, 0, 0, None, None, None, 0, 0, None, None, ws.data_ptr(), ws.numel())
    torch.cuda.synchronize()
    assert not cT.any()


def test_extreme_gates():
    """Gates at plus and minus infinity, the types' largest values and zero; a NaN stays in its unit."""
    T, H = 20, 66
    P = np.zeros((T, 1, 4 * H), np.float32)
    big = np.array([np.inf, -np.inf, 3e38, -3e38, 0.0, 100.0, -100.0, 30.0], np.float32)
    rng = np.random.default_rng(3)
    P[:] = big[rng.integers(0, len(big), P.shape)]
    P[7, 0, 5] = np.nan
    bh, cT, *_ = _run(T, 1, H, "f32", False, "tb", 0, 0, P, np.zeros((T, 1, H)), None, None, None, train=False)
    h, c, _ = oracle.scan_forward(P)
    close(bh.get(), h, 1e-5)
    close(cT.get(), c, 1e-5)
    assert np.isnan(c[0, 5]) and np.isfinite(np.delete(c[0], 5)).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_same_bits_again_and_on_another_stream(dtype):
    import torch
    T, Bn, H = 700, 2, 90
    P, dh, c0, dcT, lengths = _inputs(T, Bn, H, dtype, True, 9)
    first = [b.get() for b in _run(T, Bn, H, dtype, False, "tb", 0, 0, P, dh, c0, dcT, lengths)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        again = _run(T, Bn, H, dtype, False, "tb", 0, 0, P, dh, c0, dcT, lengths, side.cuda_stream)
    for a, b in zip(first, again):
        assert np.array_equal(a, b.get(), equal_nan=True)
