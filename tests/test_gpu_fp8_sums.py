"""The product's sums are those of fp32 whatever the type of the result and the kernel: products far below the largest of a block
count, also where the largest cancel each other."""
import numpy as np
import pytest

from lm_ops_util import Buf, DTYPE, HALF, U32, close, workspace
from oracle import lm_ops as oracle
from paper_1901_10997_amd import binding as B

pytestmark = pytest.mark.gpu

LARGEST, NEGATIVE = 126, 128 | 126          # 448 and -448


def _product(A, a_scale, W, w_scale, w_rows, out, bias=None):
    import torch
    (M, K), N = A.shape, W.shape[0]
    ld = -(-K // 16) * 16
    held = []
    for codes in (A, W):
        padded = np.full((codes.shape[0], ld), 0x7F, np.uint8)
        padded[:, :K] = codes
        held.append(torch.from_numpy(padded).to("cuda:0"))
    asd, wsd, C = Buf(a_scale.shape, data=a_scale), Buf(w_scale.shape, data=w_scale), Buf((M, N), out, 1, 1)
    bd = None if bias is None else torch.from_numpy(bias).to("cuda:0")
    ws = workspace(B.lstm_matmul_fp8_workspace_bytes(M, N, K))
    B.lstm_matmul_fp8(M, N, K, held[0].data_ptr(), ld, asd.ptr, asd.strides[0], held[1].data_ptr(), ld, wsd.ptr, wsd.strides[0], w_rows,
                      None if bd is None else bd.data_ptr(), DTYPE[out], C.ptr, C.strides[0], ws.data_ptr(), ws.numel())
    return C.get()


def _tolerance(K, out, size, want):
    """128 exact products a block one after the other at worst, two multiplications by scales, the blocks after that, the bias,
    and the rounding of the result."""
    return (128 + K / 128 + 8) * U32 * size + HALF[out] * np.abs(want)


# few rows, few tiles, tiles of 128 by 64 and of 128 by 128
SIZES = [(3, 100), (60, 333), (450, 1500), (700, 1100), (2300, 3700)]


@pytest.mark.parametrize("M,N", SIZES)
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("w_rows", [1, 128])
def test_large_products_that_cancel(M, N, out, w_rows):
    """In every block 448 * 448 - 448 * 448 beside 126 positive products of about one: their sum is the result."""
    K = 300
    rng = np.random.default_rng(M + N)
    A = rng.integers(45, 60, (M, K)).astype(np.uint8)       # 0.4 .. 1.4
    W = rng.integers(45, 60, (N, K)).astype(np.uint8)
    for k in range(0, K - 40, 128):
        A[:, k + 3], A[:, k + 37] = LARGEST, LARGEST
        W[:, k + 3], W[:, k + 37] = LARGEST, NEGATIVE
    a_scale = np.ones((M, 3), np.float32)
    w_scale = np.ones((-(-N // w_rows), 3), np.float32)
    want, size = oracle.matmul(A, a_scale, W, w_scale, w_rows)
    assert want.min() > 100
    close(_product(A, a_scale, W, w_scale, w_rows, out), want, _tolerance(K, out, size, want))


@pytest.mark.parametrize("M,N", SIZES)
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_codes_of_every_size(M, N, out):
    """Random codes: products of 2^-18 to 2^18 in one sum."""
    K = 700
    rng = np.random.default_rng(M * N)
    A, W = (np.where(c & 127 == 127, 5, c).astype(np.uint8) for c in (rng.integers(0, 256, (R, K)) for R in (M, N)))
    a_scale, w_scale = (np.exp(rng.uniform(-3, 3, s)).astype(np.float32) for s in ((M, 6), (-(-N // 128), 6)))
    want, size = oracle.matmul(A, a_scale, W, w_scale, 128)
    close(_product(A, a_scale, W, w_scale, 128, out), want, _tolerance(K, out, size, want))


SCALES = {
    # what log2 of A's and of W's scales lies around in each block of 128 columns
    "opposite": ([100, -100, 60, -60, 118, -125], [-100, 100, -70, 70, -120, 119]),
    "both small": ([-68] * 6, [-68] * 6),               # the product of two scales is below the normal numbers
    "one far larger": ([-100, -90, -110, -61, -62, -80], [119, 110, 119, 80, 80, 100]),       # .. a sum times W's above the largest
    "one far smaller": ([119, 110, 100, 61, 62, 80], [-126, -120, -126, -90, -80, -100]),
}


@pytest.mark.parametrize("M,N", SIZES)
@pytest.mark.parametrize("out,w_rows", [("f32", 1), ("f32", 128), ("bf16", 1), ("bf16", 128)])
@pytest.mark.parametrize("scales", list(SCALES))
def test_scales_far_from_one(M, N, out, w_rows, scales):
    """Scales of any size that results of ordinary size have."""
    K = 700
    rng = np.random.default_rng(M * N + len(scales))
    A, W = (rng.integers(30, 80, (R, K)).astype(np.uint8) for R in (M, N))
    if scales != "both small":          # whose results would be subnormal where the signs are mixed
        A |= (rng.integers(0, 2, (M, K)) << 7).astype(np.uint8)
    ea, ew = SCALES[scales]
    near = lambda e, R: np.ldexp(rng.uniform(1, 1.6, (R, 6)), e).astype(np.float32)  # noqa: E731
    a_scale, w_scale = near(ea, M), near(ew, -(-N // w_rows))
    want, size = oracle.matmul(A, a_scale, W, w_scale, w_rows)
    assert 2.0 ** -126 < size.min() and size.max() < 2.0 ** 126
    close(_product(A, a_scale, W, w_scale, w_rows, out), want, _tolerance(K, out, size, want))


@pytest.mark.parametrize("M,N", SIZES)
@pytest.mark.parametrize("out,w_rows", [("f32", 1), ("f32", 128), ("bf16", 1), ("bf16", 128)])
def test_large_scales_of_small_values_and_of_zeros(M, N, out, w_rows):
    """Scales whose product is beyond the largest number, of blocks in which the smallest codes meet once or not at all; a NaN among
    the scales reaches its row and its columns alone."""
    K = 200
    A, W = np.zeros((M, K), np.uint8), np.zeros((N, K), np.uint8)
    A[:, 5], A[::3, 150], W[::2, 5], W[1::2, 150] = 1, 1, 1, 129
    a_scale, w_scale = np.full((M, 2), 2.0 ** 70, np.float32), np.full((-(-N // w_rows), 2), 2.0 ** 70, np.float32)
    want, size = oracle.matmul(A, a_scale, W, w_scale, w_rows)
    assert set(np.unique(want)) == {-2.0 ** 122, 0.0, 2.0 ** 122}
    close(_product(A, a_scale, W, w_scale, w_rows, out), want, 0)
    a_scale[M // 2, 1] = w_scale[-1, 0] = np.nan
    got = _product(A, a_scale, W, w_scale, w_rows, out)
    nan = np.zeros((M, N), bool)
    nan[M // 2], nan[:, (w_scale.shape[0] - 1) * w_rows:] = True, True
    assert np.array_equal(np.isnan(got), nan)
    assert np.array_equal(got[~nan], want[~nan])


@pytest.mark.parametrize("M,N", SIZES)
@pytest.mark.parametrize("out,w_rows", [("f32", 1), ("f32", 128), ("bf16", 1), ("bf16", 128)])
def test_infinite_scales(M, N, out, w_rows):
    """They make every sum infinite, and a sum of zeros NaN, however small the sum is."""
    K = 200
    A, W = np.zeros((M, K), np.uint8), np.ones((N, K), np.uint8)
    A[:, 5], A[1::2, 5] = 1, 129                            # one product of 2^-18, of either sign, in the first block
    A[0] = 0
    a_scale, w_scale = np.full((M, 2), 2.0 ** -20, np.float32), np.full((-(-N // w_rows), 2), 2.0 ** -20, np.float32)
    a_scale[M // 2, 0] = a_scale[0, 0] = w_scale[-1, 0] = np.inf
    got = _product(A, a_scale, W, w_scale, w_rows, out)
    with np.errstate(invalid="ignore"):
        first = oracle.e4m3_decode(A[:, :128]) @ oracle.e4m3_decode(W[:, :128]).T
        want = first * a_scale[:, :1].astype(np.float64) * np.repeat(w_scale[:, 0], w_rows)[:N].astype(np.float64)
    assert np.isinf(want[M // 2]).all() and np.isnan(want[0, -1]) and np.isnan(want).sum() >= N
    assert np.array_equal(np.isnan(got), np.isnan(want))
    rest = ~np.isnan(want)
    assert np.array_equal(got[rest], want[rest])
