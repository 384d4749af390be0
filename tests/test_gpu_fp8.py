"""Quantization to e4m3 with block scales (bit for bit) and the product of such operands against the fp64 oracle."""
import numpy as np
import pytest

from lm_ops_util import Buf, DTYPE, HALF, U32, close, dev, ptr, rounded, workspace
from oracle import lm_ops as oracle
from paper_1901_10997_amd import binding as B

pytestmark = pytest.mark.gpu


def _ld(K):
    return -(-K // 16) * 16


@pytest.mark.parametrize("M,N,dtype,pad", [
    (1, 1, "f32", 0), (3, 127, "bf16", 0), (2, 128, "f32", 0), (130, 129, "bf16", 1), (129, 1500, "bf16", 0), (257, 700, "f32", 2),
    (1, 4097, "f32", 3), (300, 640, "bf16", 8),
])
@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantize(M, N, dtype, pad, block_rows):
    import torch
    rng = np.random.default_rng(M * N)
    x = rounded(rng.standard_normal((M, N)) * np.exp(rng.uniform(-8, 8, (M, 1))), dtype)
    if M > 2:
        x[1] = 0
        x[2, 0] = 1e-44 if dtype == "f32" else 1e-38
    if M > 128:
        x[128, :5] = [np.inf, -np.inf, np.nan, 0.0, 3.0]
        x[64:66] = rounded(np.full((2, N), 3e38 if block_rows == 1 else 1.0), dtype)
    bx = Buf((M, N), dtype, pad, 0, x)
    q = torch.full((M, _ld(N) + 16), 0xEE, dtype=torch.uint8, device="cuda:0")
    RB = -(-M // block_rows)
    sc = Buf((RB, -(-N // 128)), pad=1)
    B.lstm_quantize_fp8(M, N, DTYPE[dtype], block_rows, bx.ptr, bx.strides[0], q.data_ptr(), q.stride(0), sc.ptr, sc.strides[0])
    codes, scale = oracle.quantize(x, block_rows)
    assert np.array_equal(sc.get(), scale.astype(np.float64))
    got = q.cpu().numpy()
    assert (got[:, N:] == 0xEE).all()
    nan = np.isnan(x)
    assert (got[:, :N][nan] & 127 == 127).all()
    assert np.array_equal(got[:, :N][~nan], codes[~nan])


def _operand(rng, R, K, block_rows, pad=0):
    import torch
    v = rng.standard_normal((R, K)) * np.exp(0.7 * rng.standard_normal(K))
    codes, scale = oracle.quantize(v.astype(np.float32), block_rows)
    ld = _ld(K) + pad
    held = np.full((R, ld), 0x7F, np.uint8)                  # NaN behind column K
    held[:, :K] = codes
    return codes, scale, torch.from_numpy(held).to("cuda:0"), Buf(scale.shape, pad=1, data=scale)


PRODUCTS = [
    # M, N, K, out, w_block_rows, bias, pad
    (1, 1, 1, "f32", 128, False, 0), (1, 1000, 1500, "f32", 128, True, 0), (2, 17, 129, "bf16", 1, True, 16), (16, 130, 128, "f32", 1, False, 0),
    (17, 200, 257, "bf16", 128, True, 0), (33, 65, 640, "f32", 128, False, 0), (64, 300, 1000, "bf16", 1, False, 32), (65, 129, 384, "f32", 1, True, 0),
    (100, 515, 1500, "bf16", 128, True, 0), (129, 257, 700, "f32", 128, False, 16), (255, 640, 2048, "bf16", 128, False, 0),
    (257, 513, 300, "bf16", 1, True, 0), (300, 1030, 96, "f32", 128, False, 0), (700, 750, 1500, "bf16", 128, True, 0),
    (515, 1025, 127, "bf16", 128, False, 0), (1000, 300, 1025, "f32", 1, True, 0), (384, 512, 513, "bf16", 128, False, 0),
]


@pytest.mark.parametrize("M,N,K,out,w_rows,bias,pad", PRODUCTS)
def test_product(M, N, K, out, w_rows, bias, pad):
    rng = np.random.default_rng(M + 3 * N + 7 * K)
    A, a_scale, Ad, asd = _operand(rng, M, K, 1, pad)
    W, w_scale, Wd, wsd = _operand(rng, N, K, w_rows, pad)
    b = rng.standard_normal(N).astype(np.float32) if bias else None
    bd = dev(b)
    C = Buf((M, N), out, pad // 16, pad // 16)
    ws = workspace(B.lstm_matmul_fp8_workspace_bytes(M, N, K))
    call = lambda: B.lstm_matmul_fp8(M, N, K, Ad.data_ptr(), Ad.stride(0), asd.ptr, asd.strides[0], Wd.data_ptr(), Wd.stride(0), wsd.ptr,  # noqa: E731
                                     wsd.strides[0], w_rows, ptr(bd), DTYPE[out], C.ptr, C.strides[0], ws.data_ptr(), ws.numel())
    call()
    want, size = oracle.matmul(A, a_scale, W, w_scale, w_rows, b)
    # fp32: 128 exact products a block, added one after the other at worst, two multiplications by scales, the blocks after
    # that.  bf16 results may come from the matrix instruction of 8-bit operands, which sums a block's products to 2^-12 of their magnitudes
    # or better; the rounding of the result comes on top.
    tol = (128 + K / 128 + 8) * U32 * size if out == "f32" else 2.0 ** -12 * size + HALF["bf16"] * np.abs(want)
    first = C.get()
    close(first, want, tol)
    call()
    assert np.array_equal(first, C.get())


def test_no_columns_gives_the_bias_and_empty_products():
    import torch
    b = torch.randn(70, device="cuda:0")
    for M in (3, 200):
        C = Buf((M, 70))
        ws = workspace(B.lstm_matmul_fp8_workspace_bytes(M, 70, 0))
        B.lstm_matmul_fp8(M, 70, 0, None, 0, None, 0, None, 0, None, 0, 128, b.data_ptr(), B.LSTM_F32, C.ptr, 70, ws.data_ptr(), ws.numel())
        assert np.array_equal(C.get(), np.broadcast_to(b.double().cpu().numpy(), (M, 70)))
    B.lstm_matmul_fp8(0, 70, 128, None, 0, None, 0, None, 0, None, 0, 128, None, B.LSTM_F32, None, 70, ws.data_ptr(), ws.numel())


@pytest.mark.parametrize("M", [5, 150])
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_nan_stays_in_its_row_and_column(M, out):
    N, K = 200, 300
    rng = np.random.default_rng(4)
    A, a_scale, Ad, asd = _operand(rng, M, K, 1)
    W, w_scale, Wd, wsd = _operand(rng, N, K, 128)
    Ad[2, 290], Wd[150, 3] = 0x7F, 0xFF
    C = Buf((M, N), out)
    ws = workspace(B.lstm_matmul_fp8_workspace_bytes(M, N, K))
    B.lstm_matmul_fp8(M, N, K, Ad.data_ptr(), Ad.stride(0), asd.ptr, asd.strides[0], Wd.data_ptr(), Wd.stride(0), wsd.ptr, wsd.strides[0], 128,
                      None, DTYPE[out], C.ptr, N, ws.data_ptr(), ws.numel())
    got = C.get()
    nan = np.zeros((M, N), bool)
    nan[2], nan[:, 150] = True, True
    assert np.array_equal(np.isnan(got), nan)


def test_both_gradients_are_the_same_call():
    """dX = dC . W and dW = dC^T . X through transposed operands, against fp64 products of what the codes stand for."""
    import torch
    M, N, K = 160, 256, 384
    rng = np.random.default_rng(11)
    g, w, x = (rng.standard_normal(s).astype(np.float32) for s in ((M, N), (N, K), (M, K)))

    def codes(v, block_rows):
        R, K_ = v.shape
        t = torch.from_numpy(np.ascontiguousarray(v)).to("cuda:0")
        q = torch.zeros((R, _ld(K_)), dtype=torch.uint8, device="cuda:0")
        s = torch.empty((-(-R // block_rows), -(-K_ // 128)), device="cuda:0")
        B.lstm_quantize_fp8(R, K_, B.LSTM_F32, block_rows, t.data_ptr(), K_, q.data_ptr(), q.stride(0), s.data_ptr(), s.stride(0))
        return q, s

    def product(a, b, m, n, k, rows):
        C = torch.empty((m, n), device="cuda:0")
        ws = workspace(B.lstm_matmul_fp8_workspace_bytes(m, n, k))
        B.lstm_matmul_fp8(m, n, k, a[0].data_ptr(), a[0].stride(0), a[1].data_ptr(), a[1].stride(0), b[0].data_ptr(), b[0].stride(0), b[1].data_ptr(),
                          b[1].stride(0), rows, None, B.LSTM_F32, C.data_ptr(), n, ws.data_ptr(), ws.numel())
        torch.cuda.synchronize()
        return C.double().cpu().numpy()

    wq, wsc = codes(w, 128)
    wt = (wq[:, :K].t().contiguous(), wsc.t().contiguous())          # the transposed weights have the transposed scales
    gq = codes(g, 1)
    want, size = oracle.matmul(gq[0].cpu().numpy()[:, :N], gq[1].cpu().numpy(), wt[0].cpu().numpy(), wt[1].cpu().numpy(), 128)
    close(product(gq, wt, M, K, N, 128), want, 140 * U32 * size)
    gt, xt = codes(g.T, 1), codes(x.T, 1)
    want, size = oracle.matmul(gt[0].cpu().numpy()[:, :M], gt[1].cpu().numpy(), xt[0].cpu().numpy()[:, :M], xt[1].cpu().numpy(), 1)
    got = product(gt, xt, N, K, M, 1)
    close(got, want, 140 * U32 * size)
    # and near the gradient itself: two operands rounded by at most 2^-4 of each value, independently
    assert np.linalg.norm(got - g.T.astype(np.float64) @ x) <= 0.1 * np.linalg.norm(g.T @ x)
