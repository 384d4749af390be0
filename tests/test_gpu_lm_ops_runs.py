"""How the operators around the cells are run: states in place, recorded into graphs, on other streams than the default one."""
import pytest

from paper_1901_10997_amd import binding as B

pytestmark = pytest.mark.gpu

TYPE = {"f32": B.LSTM_F32, "bf16": B.LSTM_BF16}


def _torch_type(name):
    import torch
    return torch.bfloat16 if name == "bf16" else torch.float32


class Work:
    """One call of every operator, forward and back, on buffers of its own."""

    def __init__(self, T, batch, H, dtype, seed=0):
        import torch
        self.T, self.batch, self.H, self.dtype, M = T, batch, H, TYPE[dtype], T * batch
        gen = torch.Generator(device="cuda:0")
        gen.manual_seed(seed)
        self.gen, dt = gen, _torch_type(dtype)
        f = lambda *s: torch.zeros(s, device="cuda:0")  # noqa: E731
        e = lambda *s: torch.zeros(s, dtype=dt, device="cuda:0")  # noqa: E731
        self.x, self.r, self.dh, self.dsum = e(M, H), e(M, H), e(M, H), e(M, H)
        self.inputs = [self.x, self.r, self.dh, self.dsum]
        self.weight, self.c0, self.u = f(H), f(batch, H), f(M)
        self.inputs += [self.weight, self.c0, self.u]
        self.W = torch.randn((4 * H, H), generator=gen, device="cuda:0") * H ** -0.5
        ld = -(-H // 16) * 16
        byte = lambda rows, cols: torch.zeros((rows, -(-cols // 16) * 16), dtype=torch.uint8, device="cuda:0")  # noqa: E731
        kb = -(-H // 128)
        self.W8, self.Ws = byte(4 * H, H), f(-(-4 * H // 128), kb)
        self.y8, self.ys, self.h8, self.hs = byte(M, H), f(M, kb), byte(M, H), f(M, kb)
        self.sum, self.rstd = e(M, H), f(M)
        self.P, self.h, self.cT, self.states = e(M, 4 * H), e(M, H), f(batch, H), f(-(-T // B.LSTM_SCAN_STEPS), batch, H)
        self.dP, self.dc0, self.dx, self.dw = e(M, 4 * H), f(batch, H), e(M, H), f(H)
        self.logits = f(M, 4 * H)
        self.temperature, self.top_k, self.top_p, self.min_p = f(M) + 0.8, torch.full((M,), 40, dtype=torch.int32, device="cuda:0"), f(M) + 0.9, f(M) + 0.01
        self.token, self.prob, self.kept = torch.zeros(M, dtype=torch.int32, device="cuda:0"), f(M), torch.zeros(M, dtype=torch.int32, device="cuda:0")
        need = max(B.lstm_scan_workspace_bytes(T, batch, H), B.lstm_rmsnorm_workspace_bytes(M, H), B.lstm_matmul_fp8_workspace_bytes(M, 4 * H, H),
                   B.lstm_sample_workspace_bytes(M, 4 * H))
        self.ws = torch.full((need,), 0xA5, dtype=torch.uint8, device="cuda:0")
        assert ld == self.y8.shape[1]
        self.outputs = [self.y8, self.ys, self.sum, self.rstd, self.P, self.h, self.cT, self.states, self.dP, self.dc0, self.h8, self.hs, self.logits,
                        self.dx, self.dw, self.token, self.prob, self.kept]

    def draw(self):
        import torch
        for t in self.inputs:
            t.copy_(torch.rand(t.shape, generator=self.gen, device="cuda:0") if t is self.u else torch.randn(t.shape, generator=self.gen, device="cuda:0"))

    def spoil(self):
        for t in self.outputs:
            t.fill_(77)

    def run(self):
        import torch
        T, batch, H, M, d = self.T, self.batch, self.H, self.T * self.batch, self.dtype
        st, ws = torch.cuda.current_stream().cuda_stream, (self.ws.data_ptr(), self.ws.numel())
        p = lambda t: t.data_ptr()  # noqa: E731
        B.lstm_quantize_fp8(4 * H, H, B.LSTM_F32, 128, p(self.W), H, p(self.W8), self.W8.stride(0), p(self.Ws), self.Ws.stride(0), st)
        B.lstm_rmsnorm_forward(M, H, d, p(self.x), H, p(self.r), H, p(self.weight), 1e-5, p(self.sum), H, None, H, p(self.y8), self.y8.stride(0),
                               p(self.ys), self.ys.stride(0), p(self.rstd), st)
        B.lstm_matmul_fp8(M, 4 * H, H, p(self.y8), self.y8.stride(0), p(self.ys), self.ys.stride(0), p(self.W8), self.W8.stride(0), p(self.Ws),
                          self.Ws.stride(0), 128, None, d, p(self.P), 4 * H, *ws, st)
        B.lstm_scan_forward(T, batch, H, d, False, p(self.P), batch * 4 * H, 4 * H, None, p(self.c0), p(self.h), batch * H, H, p(self.cT),
                            p(self.states), *ws, st)
        B.lstm_scan_backward(T, batch, H, d, False, p(self.P), batch * 4 * H, 4 * H, None, p(self.states), p(self.dh), batch * H, H, p(self.c0),
                             p(self.dP), batch * 4 * H, 4 * H, p(self.dc0), *ws, st)
        B.lstm_quantize_fp8(M, H, d, 1, p(self.h), H, p(self.h8), self.h8.stride(0), p(self.hs), self.hs.stride(0), st)
        B.lstm_matmul_fp8(M, 4 * H, H, p(self.h8), self.h8.stride(0), p(self.hs), self.hs.stride(0), p(self.W8), self.W8.stride(0), p(self.Ws),
                          self.Ws.stride(0), 128, None, B.LSTM_F32, p(self.logits), 4 * H, *ws, st)
        B.lstm_rmsnorm_backward(M, H, d, p(self.sum), H, p(self.weight), p(self.rstd), p(self.dh), H, p(self.dsum), H, p(self.dx), H, p(self.dw),
                                *ws, st)
        B.lstm_sample(M, 4 * H, B.LSTM_F32, p(self.logits), 4 * H, None, 0, p(self.temperature), p(self.top_k), p(self.top_p), p(self.min_p),
                      p(self.u), p(self.token), p(self.prob), p(self.kept), *ws, st)

    def results(self):
        import torch
        torch.cuda.synchronize()
        return [t.clone() for t in self.outputs]


# time in one piece, time in many (the recurrence then takes two launches each way), and enough rows for the products' tiles
SIZES = [(1, 3, 100, "bf16"), (40, 2, 96, "f32"), (600, 1, 130, "bf16"), (300, 4, 256, "bf16")]


def _same(got, want):
    import torch
    return all(torch.equal(a.view(torch.uint8) if a.dtype != torch.uint8 else a, b.view(torch.uint8) if b.dtype != torch.uint8 else b)
               for a, b in zip(got, want))


@pytest.mark.parametrize("T,batch,H,dtype", SIZES)
def test_recorded_into_a_graph(T, batch, H, dtype):
    """Every replay gives what an eager run of the same inputs gives, bit for bit, with eager work between the replays."""
    import torch
    w = Work(T, batch, H, dtype)
    w.draw()
    w.run()                                     # the first use of a kernel loads it: not while recording
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        w.run()
    for _ in range(4):
        w.draw()
        w.spoil()
        w.run()
        want = w.results()
        w.spoil()
        w.ws.fill_(0x5A)
        graph.replay()
        assert _same(w.results(), want)


@pytest.mark.parametrize("T,batch,H,dtype", SIZES)
def test_on_another_stream(T, batch, H, dtype):
    """Inputs that the same stream has just been asked to write, with no wait in between; two streams side by side."""
    import torch
    works = [Work(T, batch, H, dtype, seed) for seed in (1, 2)]
    want = []
    for w in works:
        w.draw()
        w.spoil()                               # (what pads the rows of 8-bit values is not written)
        w.run()
        want.append(w.results())
    held = [[t.clone() for t in w.inputs] for w in works]
    for w in works:
        w.spoil()
        for t in w.inputs:
            t.fill_(0.25)
    torch.cuda.synchronize()
    busy = torch.randn(2000, 2000, device="cuda:0")
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in works]
    for w, keep, s in zip(works, held, streams):
        with torch.cuda.stream(s):
            for _ in range(5):
                busy @ busy                     # keeps the stream busy, so that a call on another one would read too early
            for t, k in zip(w.inputs, keep):
                t.copy_(k)
            w.run()
    for w, ok in zip(works, want):
        assert _same(w.results(), ok)


@pytest.mark.parametrize("T,batch,H,dtype,ragged", [
    (1, 3, 70, "f32", False), (64, 5, 70, "bf16", True), (700, 2, 300, "f32", True), (2100, 1, 1500, "bf16", False),
    (520, 16, 1024, "bf16", False),             # cut, and more workgroups in the gradient's last launch than run at a time
])
def test_states_in_place(T, batch, H, dtype, ragged):
    """The final state may overwrite the first one, and its gradient that of the last."""
    import torch
    torch.manual_seed(T)
    dt = _torch_type(dtype)
    P, dh = torch.randn((T, batch, 4 * H), device="cuda:0").to(dt), torch.randn((T, batch, H), device="cuda:0").to(dt)
    P[:, :, :H] += 3                            # much of the first state is left at the end
    lengths = torch.randint(0, T + 1, (batch,), device="cuda:0", dtype=torch.int32) if ragged else None
    c0, dcT = torch.randn((batch, H), device="cuda:0"), torch.randn((batch, H), device="cuda:0")
    states = torch.empty((-(-T // B.LSTM_SCAN_STEPS), batch, H), device="cuda:0")
    ws = torch.full((B.lstm_scan_workspace_bytes(T, batch, H),), 0xA5, dtype=torch.uint8, device="cuda:0")
    ptr = lambda t: None if t is None else t.data_ptr()  # noqa: E731

    def both(first, final, d_final, d_first):
        h, dP = torch.empty((T, batch, H), dtype=dt, device="cuda:0"), torch.empty_like(P)
        B.lstm_scan_forward(T, batch, H, TYPE[dtype], False, ptr(P), P.stride(0), P.stride(1), ptr(lengths), ptr(first), ptr(h), batch * H, H,
                            ptr(final), ptr(states), ptr(ws), ws.numel())
        B.lstm_scan_backward(T, batch, H, TYPE[dtype], False, ptr(P), P.stride(0), P.stride(1), ptr(lengths), ptr(states), ptr(dh), batch * H, H,
                             ptr(d_final), ptr(dP), P.stride(0), P.stride(1), ptr(d_first), ptr(ws), ws.numel())
        torch.cuda.synchronize()
        return [h, final.clone(), dP, d_first.clone()]

    want = both(c0, torch.empty_like(c0), dcT, torch.empty_like(c0))
    for _ in range(3):
        c, d = c0.clone(), dcT.clone()
        assert _same(both(c, c, d, d), want)
