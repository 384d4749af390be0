"""RMS norm of rows whose sum of squares is outside fp32, large and small, beside ordinary ones, and its outputs in the place of its
inputs, against the fp64 oracle."""
import numpy as np
import pytest

from lm_ops_util import Buf, DTYPE, HALF, U32, close, dev, ptr, rounded, workspace
from oracle import lm_ops as oracle
from paper_1901_10997_amd import binding as B

pytestmark = pytest.mark.gpu

# one wave to a row and four, one to eight granules to a lane
SHAPES = [(1030, 300), (1030, 1000), (1030, 1900), (9, 1), (9, 700), (9, 3000), (9, 8000), (9, 16384)]


@pytest.mark.parametrize("M,N", SHAPES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("eps", [0.0, 1e-30, 1e-5])
def test_rows_of_every_size(M, N, dtype, eps):
    import torch
    rng = np.random.default_rng(M + N)
    top = np.array([3e38, 1e30, 3e19, 1.0, 1e-15, 1e-18, 1e-25, 1e-34, 1e10])[np.arange(M) % 9]
    # the largest magnitude of a row is `top`, the others from a quarter of it up; times two the sum of x and its residual
    x = rounded(rng.choice([-1.0, 1.0], (M, N)) * rng.uniform(0.25, 1, (M, N)) * 0.5 * top[:, None], dtype)
    w = (1 + 0.3 * rng.standard_normal(N)).astype(np.float32)
    s = rounded(2 * x, dtype)
    bx, by, bs = Buf((M, N), dtype, 3, 1, x), Buf((M, N), dtype, 3, 1), Buf((M, N), dtype, 3, 1)
    KB, ld = -(-N // 128), -(-N // 16) * 16
    y8 = torch.zeros((M, ld), dtype=torch.uint8, device="cuda:0")
    bsc, brs, wd = Buf((M, KB)), Buf((1, M)), dev(w)
    B.lstm_rmsnorm_forward(M, N, DTYPE[dtype], bx.ptr, bx.strides[0], bx.ptr, bx.strides[0], ptr(wd), eps, bs.ptr, bs.strides[0], by.ptr, by.strides[0],
                           y8.data_ptr(), ld, bsc.ptr, bsc.strides[0], brs.ptr)
    assert np.array_equal(bs.get(), s)
    y, rstd = oracle.rmsnorm(s, w, float(np.float32(eps)))
    # as for ordinary rows (at most N / 512 roundings one after the other in a lane and ten after that; root, division and
    # products eight more), and of a subnormal rstd half a step
    rel = (N / 512 + 24) * U32
    close(brs.get()[0], rstd, rel * rstd + 2.0 ** -149, "rstd")
    # (a y below the normal numbers, of small rows beside a large eps: half a step of those)
    close(by.get(), y, (rel + 4 * U32 + HALF[dtype]) * np.abs(y) + 2.0 ** -133, "y")
    top_y = np.stack([np.abs(y[:, 128 * j:128 * j + 128]).max(1) for j in range(KB)], 1)
    want = np.maximum(top_y / 448, 2.0 ** -126)
    close(bsc.get(), want, (rel + 4 * U32) * want, "scale")
    v = y / oracle.spread(want, 1, M, N)
    close(oracle.e4m3_decode(y8.cpu().numpy()[:, :N]), v, np.maximum(2.0 ** -4 * np.abs(v), 2.0 ** -10) + 2 * (rel + 4 * U32) * np.abs(v), "y8")


@pytest.mark.parametrize("M,N", [(1030, 300), (1030, 1900), (9, 700), (9, 8000)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_outputs_in_place_of_inputs(M, N, dtype):
    """y over x and over the residual, the sum over x, dx over dy: the bits of outputs of their own."""
    import torch
    rng = np.random.default_rng(M * N)
    x, r, dy, d = (rounded(rng.standard_normal((M, N)), dtype) for _ in range(4))
    w = dev((1 + 0.3 * rng.standard_normal(N)).astype(np.float32))
    rs, ld = torch.empty(M, device="cuda:0"), -(-N // 16) * 16
    y8, scale = torch.zeros((M, ld), dtype=torch.uint8, device="cuda:0"), torch.empty((M, -(-N // 128)), device="cuda:0")

    def forward(bx, br, bs, by):
        B.lstm_rmsnorm_forward(M, N, DTYPE[dtype], bx.ptr, bx.strides[0], br.ptr, br.strides[0], ptr(w), 1e-5, bs.ptr, bs.strides[0], by.ptr, by.strides[0],
                               y8.data_ptr(), ld, scale.data_ptr(), scale.stride(0), ptr(rs))
        return bs.get(), by.get(), y8.cpu().numpy(), scale.cpu().numpy(), rs.cpu().numpy()

    new = lambda v=None: Buf((M, N), dtype, 5, 3, v)  # noqa: E731
    want = forward(new(x), new(r), new(), new())
    a, b, c = new(x), new(r), new(x)
    for got in (forward(a, new(r), new(), a), forward(new(x), b, new(), b), forward(c, new(r), c, new()), ):
        by_itself = [np.array_equal(p, q) for p, q in zip(got, want)]
        assert all(by_itself), by_itself
    both, other = new(x), new(r)
    got = forward(both, other, both, other)              # the sum over x and y over the residual at once
    assert all(np.array_equal(p, q) for p, q in zip(got, want))

    bs, bdw, ws = new(want[0]), Buf((1, N)), workspace(B.lstm_rmsnorm_workspace_bytes(M, N))

    def backward(bdy, bd, bdx):
        B.lstm_rmsnorm_backward(M, N, DTYPE[dtype], bs.ptr, bs.strides[0], ptr(w), ptr(rs), bdy.ptr, bdy.strides[0], bd.ptr, bd.strides[0], bdx.ptr, bdx.strides[0],
                                bdw.ptr, ws.data_ptr(), ws.numel())
        return bdx.get(), bdw.get()

    want = backward(new(dy), new(d), new())
    over = new(dy)
    got = backward(over, new(d), over)
    assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])
