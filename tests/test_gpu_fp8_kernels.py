"""The product of e4m3 operands through each of its kernels, with each type of result, form of scales and with a bias, at the tolerance
of fp32 sums.  Which kernel a case reaches is checked by test_fp8_kernel_cases.py."""
import numpy as np
import pytest

from lm_ops_util import Buf, DTYPE, HALF, U32, close, dev, workspace
from oracle import lm_ops as oracle
from paper_1901_10997_amd import binding as B

pytestmark = pytest.mark.gpu

# rows1: up to 16 rows; rows4: few tiles; tile2, tile4: tiles of 128 by 64 and by 128
CASES = [
    # kernel, M, N, K, out, w_block_rows, bias, (bytes in front of A, bytes between its rows), the same of W
    ("rows1", 1, 1000, 1500, "bf16", 128, True, (0, 4), (16, 4)),
    ("rows1", 16, 333, 257, "f32", 1, True, (0, 15), (0, 15)),
    ("rows1", 7, 130, 128, "bf16", 1, False, (0, 0), (0, 0)),
    ("rows1", 16, 77, 1, "f32", 128, False, (0, 15), (0, 15)),
    ("rows4", 17, 515, 700, "f32", 128, True, (16, 20), (0, 4)),
    ("rows4", 64, 3000, 1500, "bf16", 1, True, (0, 4), (0, 4)),
    ("rows4", 200, 300, 2050, "bf16", 128, False, (0, 14), (64, 14)),
    ("rows4", 129, 257, 384, "f32", 1, False, (0, 0), (0, 16)),
    ("tile2", 700, 1100, 1000, "f32", 128, True, (0, 8), (0, 24)),
    ("tile2", 700, 1100, 1000, "f32", 1, True, (0, 24), (0, 8)),
    ("tile2", 450, 2001, 900, "bf16", 128, True, (48, 12), (0, 12)),
    ("tile2", 451, 2000, 640, "bf16", 1, True, (0, 0), (0, 0)),
    ("tile2", 65, 13001, 129, "bf16", 128, False, (0, 15), (16, 15)),
    ("tile2", 1500, 1500, 300, "f32", 128, False, (0, 4), (0, 4)),
    ("tile4", 3001, 4001, 200, "f32", 128, True, (16, 8), (0, 8)),
    ("tile4", 3000, 4000, 256, "f32", 1, True, (0, 0), (0, 0)),
    ("tile4", 2900, 4100, 130, "bf16", 128, True, (0, 14), (0, 14)),
    ("tile4", 2900, 4100, 256, "bf16", 1, True, (0, 0), (32, 16)),
    ("tile4", 4100, 2900, 385, "bf16", 1, False, (0, 15), (0, 15)),
]


def operand(rng, R, K, block_rows, front, between):
    """Codes and scales, NaN in front of them, between the rows and behind the last."""
    import torch
    codes = rng.integers(0, 127, (R, K)).astype(np.uint8) | (rng.integers(0, 2, (R, K)) << 7).astype(np.uint8)
    scale = np.exp(rng.uniform(-4, 4, (-(-R // block_rows), -(-K // 128)))).astype(np.float32)
    ld = K + between
    assert ld % 16 == 0 and front % 16 == 0
    held = np.full(front + R * ld + 128, 0x7F, np.uint8)
    held[front:front + R * ld].reshape(R, ld)[:, :K] = codes
    return codes, scale, torch.from_numpy(held).to("cuda:0"), front, ld, Buf(scale.shape, pad=1, data=scale)


@pytest.mark.parametrize("kernel,M,N,K,out,w_rows,bias,a,w", CASES)
def test_product(kernel, M, N, K, out, w_rows, bias, a, w):
    rng = np.random.default_rng(M + 3 * N + 7 * K)
    A, a_scale, At, a_at, a_ld, asd = operand(rng, M, K, 1, *a)
    W, w_scale, Wt, w_at, w_ld, wsd = operand(rng, N, K, w_rows, *w)
    b = (rng.standard_normal(N) * 1e4).astype(np.float32) if bias else None
    bd = dev(b)
    C = Buf((M, N), out, 1, 1)
    ws = workspace(B.lstm_matmul_fp8_workspace_bytes(M, N, K))
    call = lambda: B.lstm_matmul_fp8(M, N, K, At.data_ptr() + a_at, a_ld, asd.ptr, asd.strides[0], Wt.data_ptr() + w_at, w_ld, wsd.ptr,  # noqa: E731
                                     wsd.strides[0], w_rows, bd.data_ptr() if bias else None, DTYPE[out], C.ptr, C.strides[0], ws.data_ptr(), ws.numel())
    call()
    want, size = oracle.matmul(A, a_scale, W, w_scale, w_rows, b)
    # 128 exact products a block one after the other at worst, multiplications by scales, the blocks after that, the bias, the result
    first = C.get()
    close(first, want, (128 + K / 128 + 8) * U32 * size + HALF[out] * np.abs(want))
    call()
    assert np.array_equal(first, C.get())


@pytest.mark.parametrize("kernel,M,N", [("rows1", 3, 1100), ("rows4", 200, 300), ("tile2", 700, 1100), ("tile4", 3000, 4000)])
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_no_columns_gives_the_bias(kernel, M, N, out):
    b = np.random.default_rng(N).standard_normal(N).astype(np.float32)
    bd, C = dev(b), Buf((M, N), out, 1, 1)
    ws = workspace(B.lstm_matmul_fp8_workspace_bytes(M, N, 0))
    for bias in (bd.data_ptr(), None):
        B.lstm_matmul_fp8(M, N, 0, None, 0, None, 0, None, 0, None, 0, 128, bias, DTYPE[out], C.ptr, C.strides[0], ws.data_ptr(), ws.numel())
        want = np.broadcast_to(b.astype(np.float64) if bias else 0.0, (M, N))
        close(C.get(), want, HALF["bf16"] * np.abs(want) if out == "bf16" else 0)
