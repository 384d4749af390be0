"""The operators on rows so far apart that their offsets pass 32 bits, and on strides behind the limit of the product's tiles: the bits of
the same rows side by side."""
import pytest

from paper_1901_10997_amd import binding as B

pytestmark = pytest.mark.gpu

FAR = (1 << 30) + 16            # elements: four rows of bf16 are 8 GiB, offsets pass 2^32 bytes from the third on, 2^31 elements too


def _rows(R, ld, dtype, values=None):
    """[R, width] rows ld apart.  What lies between them is never written, nor is it cleared."""
    import torch
    width = 0 if values is None else values.shape[1]
    t = torch.empty((R - 1) * ld + max(width, 4096), dtype=dtype, device="cuda:0")
    v = t.as_strided((R, max(width, 4096)), (ld, 1))
    if values is not None:
        v = v[:, :width]
        v.copy_(values)
    return v


def _same(a, b):
    import torch
    torch.cuda.synchronize()
    view = torch.uint8 if a.element_size() == 1 else torch.int16 if a.element_size() == 2 else torch.int32
    return torch.equal(a.contiguous().view(view), b.contiguous().view(view))


def _gen(seed=1):
    import torch
    g = torch.Generator(device="cuda:0")
    g.manual_seed(seed)
    return lambda *s: torch.randn(s, generator=g, device="cuda:0")


def test_norm_and_quantization():
    import torch
    normal, M, N = _gen(), 4, 700
    x, dy = normal(M, N).bfloat16(), normal(M, N).bfloat16()
    far = lambda v=None: _rows(M, FAR, torch.bfloat16, v)  # noqa: E731
    out = []
    for make, ld in ((lambda v=None: torch.empty_like(x) if v is None else v.clone(), N), (far, FAR)):
        a, s, y, dx, d = make(x), make(), make(), make(), make(dy)
        rstd, dw = torch.empty(M, device="cuda:0"), torch.empty(N, device="cuda:0")
        ws = torch.empty(B.lstm_rmsnorm_workspace_bytes(M, N), dtype=torch.uint8, device="cuda:0")
        B.lstm_rmsnorm_forward(M, N, B.LSTM_BF16, a.data_ptr(), ld, a.data_ptr(), ld, None, 1e-5, s.data_ptr(), ld, y.data_ptr(), ld, None, 0, None, 0, rstd.data_ptr())
        B.lstm_rmsnorm_backward(M, N, B.LSTM_BF16, s.data_ptr(), ld, None, rstd.data_ptr(), d.data_ptr(), ld, None, 0, dx.data_ptr(), ld, dw.data_ptr(), ws.data_ptr(),
                                ws.numel())
        q, scale = torch.zeros((M, 704), dtype=torch.uint8, device="cuda:0"), torch.empty((M, 6), device="cuda:0")
        B.lstm_quantize_fp8(M, N, B.LSTM_BF16, 1, a.data_ptr(), ld, q.data_ptr(), 704, scale.data_ptr(), 6)
        out.append([v[:, :N].clone() for v in (s, y, dx)] + [rstd, dw, q, scale])
        torch.cuda.synchronize()
        del a, s, y, dx, d
    assert all(_same(p, q) for p, q in zip(*out))


@pytest.mark.parametrize("T,batch", [(1, 3), (70, 3), (3, 2)])
def test_recurrence(T, batch):
    """Sequences far apart, and (three steps) steps far apart."""
    import torch
    normal, H = _gen(2), 66
    P, dh, c0 = normal(batch, T, 4 * H).bfloat16(), normal(batch, T, H).bfloat16(), normal(batch, H)
    out = []
    for far in (False, True):
        if T == 3:          # steps outermost
            lay = lambda v, w: (_rows(T, FAR, torch.bfloat16, v.transpose(0, 1).reshape(T, batch * w)) if far else v.transpose(0, 1).reshape(T, batch * w).clone())  # noqa: E731
            strides = lambda w: (FAR if far else batch * w, w)  # noqa: E731
        else:
            lay = lambda v, w: (_rows(batch, FAR, torch.bfloat16, v.reshape(batch, T * w)) if far else v.reshape(batch, T * w).clone())  # noqa: E731
            strides = lambda w: (w, FAR if far else T * w)  # noqa: E731
        p, d, h, dp = lay(P, 4 * H), lay(dh, H), lay(dh, H), lay(P, 4 * H)
        cT, dc0 = torch.empty_like(c0), torch.empty_like(c0)
        states = torch.empty((-(-T // B.LSTM_SCAN_STEPS), batch, H), device="cuda:0")
        ws = torch.empty(B.lstm_scan_workspace_bytes(T, batch, H), dtype=torch.uint8, device="cuda:0")
        B.lstm_scan_forward(T, batch, H, B.LSTM_BF16, 1, p.data_ptr(), *strides(4 * H), None, c0.data_ptr(), h.data_ptr(), *strides(H), cT.data_ptr(), states.data_ptr(),
                            ws.data_ptr(), ws.numel())
        B.lstm_scan_backward(T, batch, H, B.LSTM_BF16, 1, p.data_ptr(), *strides(4 * H), None, states.data_ptr(), d.data_ptr(), *strides(H), c0.data_ptr(), dp.data_ptr(),
                             *strides(4 * H), dc0.data_ptr(), ws.data_ptr(), ws.numel())
        out.append([h.clone(), cT, states, dp.clone(), dc0])
        torch.cuda.synchronize()
        del p, d, h, dp
    assert all(_same(a, b) for a, b in zip(*out))


def test_draw():
    import torch
    normal, M, V = _gen(3), 4, 3000
    logits = normal(M, V).bfloat16()
    allowed = (normal(M, V) < 1).to(torch.uint8)
    u, p = torch.rand(M, device="cuda:0"), torch.full((M,), 0.9, device="cuda:0")
    out = []
    for far in (False, True):
        l, a = (_rows(M, FAR, torch.bfloat16, logits), _rows(M, 4 * FAR, torch.uint8, allowed)) if far else (logits, allowed)
        token, prob, kept = torch.empty(M, dtype=torch.int32, device="cuda:0"), torch.empty(M, device="cuda:0"), torch.empty(M, dtype=torch.int32, device="cuda:0")
        ws = torch.empty(256, dtype=torch.uint8, device="cuda:0")
        B.lstm_sample(M, V, B.LSTM_BF16, l.data_ptr(), l.stride(0), a.data_ptr(), a.stride(0), None, None, p.data_ptr(), None, u.data_ptr(), token.data_ptr(), prob.data_ptr(),
                      kept.data_ptr(), ws.data_ptr(), ws.numel())
        out.append([token, prob, kept])
        torch.cuda.synchronize()
        del l, a
    assert all(_same(a, b) for a, b in zip(*out))


@pytest.mark.parametrize("M,N,a_ld,w_ld,scale_ld,c_ld", [
    (200, 300, 1 << 22, 1 << 22, 8, 300),                   # the kernel for few rows, operands of 800 MB and more
    (200, 6500, (1 << 23) - 16, 400, 8, 6500),              # tiles, at the largest stride that they take
    (200, 6500, 1 << 23, 400, 8, 6500),                     # .. and behind it
    (100, 7000, 400, 400, (1 << 21) - 1, 7000),             # the same of the scales' rows
    (100, 7000, 400, 400, 1 << 21, 7000),
    (200, 6500, 400, 400, 8, 1 << 25),                      # results over 12 GiB
])
def test_product(M, N, a_ld, w_ld, scale_ld, c_ld):
    import torch
    K = 400
    g = torch.Generator(device="cuda:0")
    g.manual_seed(4)
    A, W = (torch.randint(0, 120, (R, K), generator=g, device="cuda:0").to(torch.uint8) for R in (M, N))
    a_scale, w_scale = (torch.rand((R, 4), generator=g, device="cuda:0") for R in (M, -(-N // 128)))
    out = []
    for far in (False, True):
        a, w, s = (_rows(M, a_ld, torch.uint8, A), _rows(N, w_ld, torch.uint8, W), _rows(M, scale_ld, torch.float32, a_scale)) if far else (A, W, a_scale)
        c = _rows(M, c_ld, torch.bfloat16, torch.zeros((M, N), dtype=torch.bfloat16, device="cuda:0")) if far else torch.empty((M, N), dtype=torch.bfloat16, device="cuda:0")
        ws = torch.empty(256, dtype=torch.uint8, device="cuda:0")
        B.lstm_matmul_fp8(M, N, K, a.data_ptr(), a.stride(0), s.data_ptr(), s.stride(0), w.data_ptr(), w.stride(0), w_scale.data_ptr(), 4, 128, None, B.LSTM_BF16,
                          c.data_ptr(), c.stride(0), ws.data_ptr(), ws.numel())
        out.append(c.clone())
        torch.cuda.synchronize()
        del a, w, s, c
    got, want = out[1].double(), out[0].double()
    # another kernel may have taken it: fp32 sums in another order (128 + 4 + 8 roundings each, relative to positive sums), then a step of bf16
    assert bool(((got - want).abs() <= (2 * 140 * 2.0 ** -24 + 2 * 2.0 ** -8) * want.abs()).all())
