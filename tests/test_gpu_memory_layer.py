"""The delta rule, the scores and the distillation loss as they are used: a layer with a matrix memory between the library's norms, its logits scored and
compared with a teacher's, forward, back, and token by token in a graph.

    q, k = norm per head of Q, K (weight key_dim^-1/2: length 1)     o = delta rule(q, k, V)     logits = o W^T     loss = distillation + likelihood
"""
import numpy as np
import pytest

from paper_1901_10997_amd import binding as B
from tests.lm_ops_util import dev, ptr, workspace

pytestmark = pytest.mark.gpu
EPS = 1e-6


class Layer:
    """Everything in fp32; W multiplied by torch, which only carries memory and this plain product here."""

    def __init__(self, T, batch, heads, dim, words, seed=0):
        import torch
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        self.T, self.batch, self.heads, self.dim, self.words = T, batch, heads, dim, words
        self.raw = torch.randn((T, batch, 3 * heads * dim), generator=gen, device="cuda")       # Q, K, V side by side
        self.beta = torch.rand((T, batch, heads), generator=gen, device="cuda")
        self.g = -torch.rand((T, batch, heads), generator=gen, device="cuda") * 0.2
        self.W = torch.randn((words, heads * dim), generator=gen, device="cuda")
        self.unit = torch.full((dim,), dim ** -0.5, device="cuda")
        self.token = torch.randint(0, words, (T, batch), generator=gen, device="cuda", dtype=torch.int32)
        self.top = torch.stack([torch.randperm(words, generator=gen, device="cuda")[:8] for _ in range(T * batch)]).to(torch.int32)
        self.top_logit = torch.randn((T * batch, 8), generator=gen, device="cuda")
        self.teacher_lse = torch.logsumexp(self.top_logit, 1) + 0.3
        self.n = heads * dim

    def stream(self):
        import torch
        return torch.cuda.current_stream().cuda_stream

    def norm(self, x, y, rstd):
        M = x.numel() // self.dim
        B.lstm_rmsnorm_forward(M, self.dim, 0, ptr(x), self.dim, None, 0, ptr(self.unit), EPS, None, 0, ptr(y), self.dim, None, 0, None, 0, ptr(rstd), self.stream())

    def norm_back(self, x, rstd, dy):
        import torch
        M, dx = x.numel() // self.dim, torch.empty_like(x)
        ws = workspace(B.lstm_rmsnorm_workspace_bytes(M, self.dim))
        B.lstm_rmsnorm_backward(M, self.dim, 0, ptr(x), self.dim, ptr(self.unit), ptr(rstd), ptr(dy), self.dim, None, 0, ptr(dx), self.dim, None, ptr(ws), ws.numel(),
                                self.stream())
        return dx

    def delta_inputs(self, T, q, k, v, g, beta):
        rows = lambda t: (ptr(t), t.stride(0), t.stride(1))      # noqa: E731
        return (T, self.batch, self.heads, self.heads, self.dim, self.dim, 0, *rows(q), *rows(k), *rows(v), *rows(g), *rows(beta), None, 1.0)

    def run(self):
        """loss per position, and the gradients of Q, K, V, g, beta and W."""
        import torch
        T, batch, n, M = self.T, self.batch, self.n, self.T * self.batch
        Q, K, V = (self.raw[..., i * n:(i + 1) * n] for i in range(3))
        Qc, Kc = Q.contiguous(), K.contiguous()
        q, k = torch.empty_like(Qc), torch.empty_like(Kc)
        rq, rk = torch.empty(M * self.heads, device="cuda"), torch.empty(M * self.heads, device="cuda")
        self.norm(Qc, q, rq)
        self.norm(Kc, k, rk)
        o, ST = torch.empty((T, batch, n), device="cuda"), torch.empty((batch, self.heads, self.dim, self.dim), device="cuda")
        states = torch.empty((-(-T // 64), *ST.shape), device="cuda")
        ws = workspace(B.lstm_delta_workspace_bytes(T, batch, self.heads, self.heads, self.dim, self.dim, True))
        inputs = self.delta_inputs(T, q, k, V, self.g, self.beta)
        B.lstm_delta_forward(*inputs, None, ptr(o), o.stride(0), o.stride(1), ptr(ST), ptr(states), ptr(ws), ws.numel(), self.stream())
        logits = (o.view(M, n) @ self.W.T).contiguous()
        lp, stats = torch.empty(M, device="cuda"), torch.empty((M, 4), device="cuda")
        loss, stats2 = torch.empty(M, device="cuda"), torch.empty((M, 4), device="cuda")
        sw = workspace(max(B.lstm_logprobs_workspace_bytes(M, self.words), B.lstm_distill_workspace_bytes(M, self.words, 8)))
        rows = (M, self.words, 0, ptr(logits), self.words, None, 0, ptr(self.token))
        B.lstm_logprobs_forward(*rows, ptr(lp), None, None, ptr(stats), 0, None, None, ptr(sw), sw.numel(), self.stream())
        lists = (M, self.words, 8, 0, ptr(logits), self.words, ptr(self.top), 8, ptr(self.top_logit), 8, ptr(self.teacher_lse), 1.5)
        B.lstm_distill_forward(*lists, ptr(loss), ptr(stats2), ptr(sw), sw.numel(), self.stream())
        d1, d2 = torch.empty_like(logits), torch.empty_like(logits)
        minus, one = torch.full((M,), -1.0, device="cuda"), torch.ones(M, device="cuda")
        B.lstm_logprobs_backward(*rows, ptr(stats), ptr(minus), None, ptr(d1), self.words, self.stream())
        B.lstm_distill_backward(*lists, ptr(stats2), ptr(one), ptr(d2), self.words, self.stream())
        dlogits = d1 + d2
        dW, do = dlogits.T.contiguous() @ o.view(M, n), (dlogits @ self.W).view(T, batch, n)
        dq, dk, dv, dg, db = (torch.empty_like(x) for x in (q, k, q, self.g, self.beta))
        rs = lambda t: (ptr(t), t.stride(0), t.stride(1))      # noqa: E731
        B.lstm_delta_backward(*inputs, ptr(states), *rs(do), None, *rs(dq), *rs(dk), *rs(dv), *rs(dg), *rs(db), None, ptr(ws), ws.numel(), self.stream())
        dQ, dK = self.norm_back(Qc, rq, dq), self.norm_back(Kc, rk, dk)
        return loss - lp, dict(Q=dQ, K=dK, V=dv, g=dg, beta=db, W=dW), (o, ST, logits)

    def plain(self):
        """The same in 64 bits on the CPU, its gradients by torch."""
        import torch
        raw, beta, g, W = (x.double().cpu().requires_grad_() for x in (self.raw, self.beta, self.g, self.W))
        T, batch, H, D = self.T, self.batch, self.heads, self.dim
        Q, K, V = (raw[..., i * self.n:(i + 1) * self.n].reshape(T, batch, H, D) for i in range(3))
        unit = lambda x: x * (x.square().mean(-1, keepdim=True) + EPS).rsqrt() * D ** -0.5        # noqa: E731
        q, k, S, o = unit(Q), unit(K), torch.zeros((batch, H, D, D), dtype=torch.float64), []
        for t in range(T):
            S = g[t].exp()[..., None, None] * S
            u = beta[t][..., None] * (V[t] - (k[t][..., None] * S).sum(2))
            S = S + k[t][..., None] * u[..., None, :]
            o.append((q[t][..., None] * S).sum(2))
        logits = torch.stack(o).reshape(T * batch, -1) @ W.T
        likelihood = torch.log_softmax(logits, 1).gather(1, self.token.cpu().long().view(-1, 1))[:, 0]
        heat = 1.5
        s, top = torch.softmax(logits / heat, 1), self.top.cpu().long()
        t = (self.top_logit.double().cpu() / heat - self.teacher_lse.double().cpu()[:, None]).exp()
        mine, t_rest = s.gather(1, top), 1 - t.sum(1)
        distilled = heat ** 2 * ((t * (t / mine).log()).sum(1) + t_rest * (t_rest / (1 - mine.sum(1))).log())
        loss = distilled - likelihood
        loss.sum().backward()
        n = self.n
        return loss.detach(), dict(Q=raw.grad[..., :n], K=raw.grad[..., n:2 * n], V=raw.grad[..., 2 * n:], g=g.grad, beta=beta.grad, W=W.grad)


def _off(a, b):
    return float((a.double().cpu() - b).norm() / b.norm())


def test_loss_and_gradients_through_all_of_it():
    layer = Layer(140, 2, 3, 20, 300)
    loss, grad, _ = layer.run()
    want, wanted = layer.plain()
    # fp32 throughout: a value passes through a norm, T = 140 corrections and products of up to 300 terms and the same way back.  Independent
    # roundings of 2^-24 each add like the root of their number: 2^-24 sqrt(2 (140 + 300 + 60 + 20)) = 2e-6; the softmax's arguments, up to 30, take theirs
    # with them, 2^-24 30 = 2e-6; eight times their sum.
    assert _off(loss, want) < 3.2e-5
    for k, v in wanted.items():
        assert _off(grad[k], v) < 3.2e-5, (k, _off(grad[k], v))


def test_recorded_steps_are_those_of_the_whole():
    """The layer's last tokens one by one from the state behind the first, in a recorded graph that is replayed."""
    import torch
    layer = Layer(100, 3, 2, 64, 50, seed=1)
    _, _, (o, ST, logits) = layer.run()
    n, first = layer.n, 90
    now = {k: torch.empty((1, 3, n), device="cuda") for k in "QKVqko"}
    now.update(g=torch.empty((1, 3, 2), device="cuda"), beta=torch.empty((1, 3, 2), device="cuda"), r=torch.empty(6, device="cuda"))
    state = torch.zeros_like(ST)
    ws = workspace(max(256, B.lstm_delta_workspace_bytes(1, 3, 2, 2, 64, 64)))
    score_ws = workspace(B.lstm_logprobs_workspace_bytes(3, 50, 4))
    token, lp, rank, top, top_lp = (torch.empty(s, dtype=t, device="cuda") for s, t in (((3,), torch.int32), ((3,), torch.float32), ((3,), torch.int32),
                                                                                         ((3, 4), torch.int32), ((3, 4), torch.float32)))
    out = torch.empty((3, 50), device="cuda")
    WT = layer.W.T.contiguous()

    def step():
        layer.norm(now["Q"], now["q"], now["r"])
        layer.norm(now["K"], now["k"], now["r"])
        B.lstm_delta_forward(*layer.delta_inputs(1, now["q"], now["k"], now["V"], now["g"], now["beta"]), ptr(state), ptr(now["o"]), n, n, ptr(state), None, ptr(ws),
                             ws.numel(), layer.stream())
        torch.mm(now["o"].view(3, n), WT, out=out)
        B.lstm_logprobs_forward(3, 50, 0, ptr(out), 50, None, 0, ptr(token), ptr(lp), ptr(rank), None, None, 4, ptr(top), ptr(top_lp), ptr(score_ws), score_ws.numel(),
                                layer.stream())

    def put(t):
        for i, k in enumerate("QKV"):
            now[k].copy_(layer.raw[t:t + 1, :, i * n:(i + 1) * n])
        now["g"].copy_(layer.g[t:t + 1])
        now["beta"].copy_(layer.beta[t:t + 1])
        token.copy_(layer.token[t])

    put(0)
    token.zero_()
    step()          # everything the library sets up once, in front of the recording
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        step()
    state.zero_()
    for t in range(100):
        put(t)
        graph.replay()
        torch.cuda.synchronize()
        # two ways of summing 100 corrections of 64 terms: 8 x 2^-24 sqrt(100 (64 + 192)), relative to the largest state and value
        tol = 8 * 2.0 ** -24 * np.sqrt(100 * 256) * 12
        assert float((now["o"][0] - o[t]).abs().max()) < tol
        if t >= first:
            want = torch.log_softmax(out.double(), 1)
            assert float((lp.double() - want.gather(1, token.long()[:, None])[:, 0]).abs().max()) < 1e-5
            assert bool((top[:, 0] == out.argmax(1)).all()) and bool((rank >= 0).all())
    assert float((state - ST).abs().max()) < 8 * 2.0 ** -24 * np.sqrt(100 * 256) * 12
