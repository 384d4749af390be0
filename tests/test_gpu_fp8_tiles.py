"""The product of e4m3 operands at sizes that its tiled kernels take, against the fp64 oracle: rows that start on lines of 128
bytes and rows that do not, for either operand, large and small tiles, every type of result and of scales."""
import numpy as np
import pytest

from lm_ops_util import Buf, DTYPE, HALF, U32, close, workspace
from oracle import lm_ops as oracle
from paper_1901_10997_amd import binding as B

pytestmark = pytest.mark.gpu

CASES = [
    # M, N, K, out, w_block_rows, (bytes in front of A, bytes between its rows), the same of W
    (450, 1100, 640, "bf16", 128, (0, 0), (0, 0)),              # small tiles, whole lines
    (700, 1100, 1000, "f32", 1, (16, 8), (0, 24)),
    (700, 1030, 500, "bf16", 1, (0, 12), (48, 12)),
    (450, 1100, 7300, "bf16", 128, (0, 12), (0, 12)),           # .. and blocks in two lines
    (450, 1100, 7300, "bf16", 1, (112, 28), (16, 44)),
    (515, 1151, 7296, "bf16", 128, (0, 0), (16, 0)),            # lines of A whole, every row of W sixteen bytes behind
    (515, 1151, 7296, "bf16", 128, (80, 16), (0, 0)),
    (1000, 2100, 2049, "bf16", 128, (0, 15), (64, 63)),
    (2300, 3700, 256, "bf16", 128, (0, 0), (0, 0)),             # large tiles
    (2300, 3700, 200, "f32", 128, (16, 8), (0, 8)),
    (2300, 3700, 130, "f32", 1, (0, 14), (0, 14)),
    (2305, 3701, 1027, "bf16", 128, (0, 13), (32, 13)),
    (2305, 3701, 1152, "bf16", 1, (96, 48), (0, 0)),
]


def _operand(rng, R, K, block_rows, front, between):
    import torch
    v = rng.standard_normal((R, K)).astype(np.float32) * np.exp(0.7 * rng.standard_normal(K)).astype(np.float32)
    codes, scale = oracle.quantize(v, block_rows)
    ld = K + between
    assert ld % 16 == 0
    held = np.full(front + R * ld + 128, 0x7F, np.uint8)        # NaN in front, behind column K and behind the last row
    held[front:front + R * ld].reshape(R, ld)[:, :K] = codes
    t = torch.from_numpy(held).to("cuda:0")
    assert t.data_ptr() % 128 == 0
    return codes, scale, t, t.data_ptr() + front, ld, Buf(scale.shape, pad=1, data=scale)


@pytest.mark.parametrize("M,N,K,out,w_rows,a,w", CASES)
def test_product(M, N, K, out, w_rows, a, w):
    rng = np.random.default_rng(M + 3 * N + 7 * K)
    A, a_scale, At, a_ptr, a_ld, asd = _operand(rng, M, K, 1, *a)
    W, w_scale, Wt, w_ptr, w_ld, wsd = _operand(rng, N, K, w_rows, *w)
    C = Buf((M, N), out, 1, 1)
    ws = workspace(B.lstm_matmul_fp8_workspace_bytes(M, N, K))
    call = lambda: B.lstm_matmul_fp8(M, N, K, a_ptr, a_ld, asd.ptr, asd.strides[0], w_ptr, w_ld, wsd.ptr, wsd.strides[0], w_rows, None,  # noqa: E731
                                     DTYPE[out], C.ptr, C.strides[0], ws.data_ptr(), ws.numel())
    call()
    want, size = oracle.matmul(A, a_scale, W, w_scale, w_rows, None)
    # as for the small sizes: fp32 128 exact products a block one after the other at worst, two multiplications by scales, the
    # blocks after that; bf16 a block's products to 2^-12 of their magnitudes, and the rounding of the result
    tol = (128 + K / 128 + 8) * U32 * size if out == "f32" else 2.0 ** -12 * size + HALF["bf16"] * np.abs(want)
    first = C.get()
    close(first, want, tol)
    call()
    assert np.array_equal(first, C.get())
    assert At.numel() and Wt.numel()        # the operands' memory is theirs until here


@pytest.mark.parametrize("M,N,K,out", [(450, 1100, 7300, "bf16"), (700, 1100, 300, "f32"), (2300, 3700, 300, "bf16")])
def test_nan_stays_in_its_row_and_column(M, N, K, out):
    rng = np.random.default_rng(5)
    _, _, At, a_ptr, a_ld, asd = _operand(rng, M, K, 1, 0, -K % 16)
    _, _, Wt, w_ptr, w_ld, wsd = _operand(rng, N, K, 128, 0, -K % 16)
    At[(M - 2) * a_ld + K - 1], Wt[(N - 3) * w_ld] = 0x7F, 0xFF
    C = Buf((M, N), out)
    ws = workspace(B.lstm_matmul_fp8_workspace_bytes(M, N, K))
    B.lstm_matmul_fp8(M, N, K, a_ptr, a_ld, asd.ptr, asd.strides[0], w_ptr, w_ld, wsd.ptr, wsd.strides[0], 128, None, DTYPE[out], C.ptr, N,
                      ws.data_ptr(), ws.numel())
    nan = np.zeros((M, N), bool)
    nan[M - 2], nan[:, N - 3] = True, True
    assert np.array_equal(np.isnan(C.get()), nan)
