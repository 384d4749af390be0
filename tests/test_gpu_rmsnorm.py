"""RMS norm with residual and 8-bit output, and its gradient, against the fp64 oracle."""
import numpy as np
import pytest

from lm_ops_util import Buf, DTYPE, HALF, U32, close, dev, ptr, rounded, workspace
from oracle import lm_ops as oracle
from paper_1901_10997_amd import binding as B

pytestmark = pytest.mark.gpu

SHAPES = [
    # M, N, dtype, pad, offset
    (1, 1, "f32", 0, 0), (1, 1500, "bf16", 0, 0), (3, 127, "bf16", 0, 0), (2, 128, "f32", 0, 0), (5, 129, "f32", 3, 1),
    (1100, 257, "bf16", 1, 0), (1030, 600, "bf16", 0, 0), (1025, 1200, "f32", 0, 4), (1027, 2048, "bf16", 8, 8), (7, 2049, "bf16", 0, 0),
    (2, 4100, "f32", 0, 0), (3, 8192, "bf16", 0, 0), (2, 16384, "f32", 0, 0), (3, 9001, "bf16", 0, 3), (2050, 64, "f32", 0, 0),
    (1500, 1001, "f32", 0, 0),
]


def _rows(rng, M, N, dtype, size=1.0):
    return rounded(rng.standard_normal((M, N)) * size * np.exp(0.5 * rng.standard_normal(N)), dtype)


def _eight(M, N):
    import torch
    ld = -(-N // 16) * 16 + 16
    return torch.full((M, ld), 0xEE, dtype=torch.uint8, device="cuda:0"), ld


@pytest.mark.parametrize("M,N,dtype,pad,off", SHAPES)
@pytest.mark.parametrize("residual", [True, False])
def test_forward(M, N, dtype, pad, off, residual):
    rng = np.random.default_rng(M + N)
    x, w = _rows(rng, M, N, dtype), (1 + 0.3 * rng.standard_normal(N)).astype(np.float32)
    r = _rows(rng, M, N, dtype, 2.0) if residual else None
    if M > 2:
        x[1] = 0
        if residual:
            r[1] = 0
    eps = 1e-5
    bx, bs, by = Buf((M, N), dtype, pad, off, x), Buf((M, N), dtype, pad, off), Buf((M, N), dtype, pad, off)
    br = Buf((M, N), dtype, pad, off, r) if residual else None
    y8, ld = _eight(M, N)
    KB = -(-N // 128)
    bsc, brs = Buf((M, KB), pad=2), Buf((1, M))
    wd = dev(w)
    B.lstm_rmsnorm_forward(M, N, DTYPE[dtype], bx.ptr, bx.strides[0], br.ptr if residual else None, br.strides[0] if residual else 0, ptr(wd), eps,
                           bs.ptr, bs.strides[0], by.ptr, by.strides[0], y8.data_ptr(), ld, bsc.ptr, bsc.strides[0], brs.ptr)
    # the sum is one fp32 addition of values of the type, rounded to it
    s = rounded(np.float32(x) + np.float32(r), dtype) if residual else x
    assert np.array_equal(bs.get(), s)
    y, rstd = oracle.rmsnorm(s, w, eps)
    # a sum of N squares in fp32: at most N halves of a step, N / 512 of them one after the other in a lane and ten after that;
    # division, root and reciprocal four more
    rel = (N / 512 + 20) * U32
    close(brs.get()[0], rstd, rel * rstd, "rstd")
    close(by.get(), y, (rel + 4 * U32 + HALF[dtype]) * np.abs(y), "y")
    # scales: the block's largest y over 448; codes: half a step of e4m3 (2^-4 relative, 2^-10 below its normals) of y / scale
    top = np.stack([np.abs(y[:, 128 * j:128 * j + 128]).max(1) for j in range(KB)], 1)
    want = np.maximum(top / 448, 2.0 ** -126)
    scale = bsc.get()
    close(scale, want, (rel + 4 * U32) * want, "scale")
    codes = y8.cpu().numpy()
    assert (codes[:, N:] == 0xEE).all()
    v = y / oracle.spread(want, 1, M, N)
    close(oracle.e4m3_decode(codes[:, :N]), v, np.maximum(2.0 ** -4 * np.abs(v), 2.0 ** -10) + 2 * (rel + 4 * U32) * np.abs(v), "y8")


@pytest.mark.parametrize("M,N,dtype,pad,off", SHAPES)
@pytest.mark.parametrize("extra", [True, False])
def test_gradient(M, N, dtype, pad, off, extra):
    rng = np.random.default_rng(2 * M + N)
    s, dy, w = _rows(rng, M, N, dtype), _rows(rng, M, N, dtype, 0.3), (1 + 0.3 * rng.standard_normal(N)).astype(np.float32)
    d = _rows(rng, M, N, dtype, 0.5) if extra else None
    rstd = (1 / np.sqrt((s * s).mean(1) + 1e-5)).astype(np.float32)
    bs, bdy, bdx = Buf((M, N), dtype, pad, off, s), Buf((M, N), dtype, pad, off, dy), Buf((M, N), dtype, pad, off)
    bd = Buf((M, N), dtype, pad, off, d) if extra else None
    bdw, wd, rd = Buf((1, N)), dev(w), dev(rstd)
    ws = workspace(B.lstm_rmsnorm_workspace_bytes(M, N))
    args = lambda dx: (M, N, DTYPE[dtype], bs.ptr, bs.strides[0], ptr(wd), ptr(rd), bdy.ptr, bdy.strides[0], bd.ptr if extra else None,  # noqa: E731
                       bd.strides[0] if extra else 0, dx.ptr, dx.strides[0], bdw.ptr, ws.data_ptr(), ws.numel())
    B.lstm_rmsnorm_backward(*args(bdx))
    dx, dw = oracle.rmsnorm_backward(s, w, rstd, dy, d)
    # each term by its own roundings, and the inner sum as in the forward, of terms of both signs: relative to their magnitudes
    g, xh = np.abs(dy * w), np.abs(s * rstd[:, None].astype(np.float64))
    size = rstd[:, None] * (g + xh * (g * xh).mean(1, keepdims=True))
    close(bdx.get(), dx, (N / 512 + 24) * U32 * size + 2 * U32 * np.abs(dx) + HALF[dtype] * np.abs(dx), "dx")
    close(bdw.get()[0], dw, (M / 1 + 16) * U32 * (np.abs(dy) * xh).sum(0) if M < 64 else (M / 8 + 64) * U32 * (np.abs(dy) * xh).sum(0), "dw")
    once = bdx.t.clone()
    if extra:                       # in place of what came from elsewhere
        B.lstm_rmsnorm_backward(*args(bd))
        assert np.array_equal(bd.get(), once.double().cpu().numpy())


def test_gradient_against_differences():
    M, N = 5, 40
    rng = np.random.default_rng(1)
    s, w, dy = rng.standard_normal((M, N)), 1 + 0.3 * rng.standard_normal(N), rng.standard_normal((M, N))
    s, w, dy = (np.float32(v) for v in (s, w, dy))
    rstd = (1 / np.sqrt((np.float64(s) ** 2).mean(1) + 1e-5)).astype(np.float32)
    bs, bdy, bdx, bdw, wd, rd = Buf((M, N), data=s), Buf((M, N), data=dy), Buf((M, N)), Buf((1, N)), dev(w), dev(rstd)
    ws = workspace(B.lstm_rmsnorm_workspace_bytes(M, N))
    B.lstm_rmsnorm_backward(M, N, B.LSTM_F32, bs.ptr, N, ptr(wd), ptr(rd), bdy.ptr, N, None, 0, bdx.ptr, N, bdw.ptr, ws.data_ptr(), ws.numel())
    value = lambda s, w: (oracle.rmsnorm(s, w, 1e-5)[0] * dy).sum()  # noqa: E731
    for _ in range(3):
        vs, vw, step = rng.standard_normal((M, N)), rng.standard_normal(N), 1e-5
        want = (value(s + step * vs, w + step * vw) - value(s - step * vs, w - step * vw)) / (2 * step)
        got = (bdx.get() * vs).sum() + (bdw.get()[0] * vw).sum()
        assert abs(got - want) <= 1e-4 * np.sqrt((bdx.get() ** 2).sum() + (bdw.get() ** 2).sum())


def test_rows_do_not_see_each_other_and_none():
    import torch
    M, N = 6, 300
    x = torch.randn((M, N), device="cuda:0")
    x[1, 7], x[3, 200], x[4] = float("nan"), float("inf"), 0
    y = torch.empty_like(x)
    y8, ld = _eight(M, N)
    scale = torch.empty((M, 3), device="cuda:0")
    B.lstm_rmsnorm_forward(M, N, B.LSTM_F32, x.data_ptr(), N, None, 0, None, 1e-5, None, 0, y.data_ptr(), N, y8.data_ptr(), ld, scale.data_ptr(), 3, None)
    torch.cuda.synchronize()
    assert y[1].isnan().all() and (y8[1, :N].cpu() & 127 == 127).all()
    assert y[3, 200].isnan() and not y[3, :200].any() and y8[3, 200].item() & 127 == 127 and not (y8[3, :200] & 127).any()
    assert not y[4].any() and not (y8[4, :N] & 127).any() and (scale[4] == 2.0 ** -126).all()
    want, _ = oracle.rmsnorm(x.double().cpu().numpy()[[0, 2, 5]], None, 1e-5)
    close(y.double().cpu().numpy()[[0, 2, 5]], want, 32 * U32 * np.abs(want))
    dw = torch.full((N,), 5.0, device="cuda:0")
    ws = workspace(B.lstm_rmsnorm_workspace_bytes(0, N))
    B.lstm_rmsnorm_forward(0, N, B.LSTM_F32, None, N, None, 0, None, 1e-5, None, 0, None, 0, None, 0, None, 0, None)
    B.lstm_rmsnorm_backward(0, N, B.LSTM_F32, None, N, None, None, None, N, None, 0, None, N, dw.data_ptr(), ws.data_ptr(), ws.numel())
    torch.cuda.synchronize()
    assert not dw.any()


def test_in_place_residual_and_same_bits():
    import torch
    M, N = 1200, 1500
    g = torch.Generator(device="cuda:0").manual_seed(1)
    x = torch.randn((M, N), device="cuda:0", generator=g).bfloat16()
    r = torch.randn((M, N), device="cuda:0", generator=g).bfloat16()
    outs = []
    for _ in range(2):
        res, y = r.clone(), torch.empty_like(x)
        B.lstm_rmsnorm_forward(M, N, B.LSTM_BF16, x.data_ptr(), N, res.data_ptr(), N, None, 1e-5, res.data_ptr(), N, y.data_ptr(), N, None, 0, None, 0, None)
        outs.append((res, y))
    torch.cuda.synchronize()
    assert torch.equal(outs[0][0], (x.float() + r.float()).bfloat16())
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
