"""A language model of gated linear recurrences that runs the library's language-model operators together: it reads a prompt,
writes on from it token by token, and learns.

    x = embedding[token]
    a block:   s = x + r             y = norm(s)          8-bit values with scales, in one launch   (lstm_rmsnorm_forward)
               P = y W_in^T + b                           product of 8-bit operands                 (lstm_matmul_fp8)
               h = recurrence(P)                          the cell without W_h                      (lstm_scan_forward)
               r = quantize(h) W_out^T                    added in front of the next norm           (lstm_quantize_fp8, lstm_matmul_fp8)
    logits = norm(x + r) W_vocabulary^T                   token = draw(logits, u)                   (lstm_sample)

Learning goes back through the same operators: lstm_scan_backward, lstm_rmsnorm_backward, and each product's two gradients as
products of transposed 8-bit operands.  torch holds the memory, gathers the embeddings, and computes the loss of the logits.

    python3 examples/recurrent_lm.py                          two blocks of 1500 units, 10 000 words
    python3 examples/recurrent_lm.py --train 50 --units 256 --words 500
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1901_10997_amd import binding as B  # noqa: E402

EPS = 1e-5
TYPE = {torch.float32: B.LSTM_F32, torch.bfloat16: B.LSTM_BF16}


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _ptr(t):
    return None if t is None else t.data_ptr()


def _blocks(n):
    return -(-n // 128)


class Eight:
    """Matrix of e4m3 codes with a scale for block_rows rows and 128 columns.  Rows start on lines of 128 bytes, which the
    product reads fastest."""

    def __init__(self, rows, cols, block_rows=1):
        self.rows, self.cols, self.block_rows = rows, cols, block_rows
        self.codes = torch.zeros((rows, 128 * _blocks(cols)), dtype=torch.uint8, device="cuda")
        self.scale = torch.empty((-(-rows // block_rows), _blocks(cols)), device="cuda")

    def transposed(self):
        """Of a matrix with blocks of 128 by 128: the transposed codes have the transposed scales."""
        assert self.block_rows == 128
        t = Eight(self.cols, self.rows, 128)
        t.codes[:, :self.rows].copy_(self.codes[:, :self.cols].t())
        t.scale.copy_(self.scale.t())
        return t


def quantize(x, block_rows=1, out=None):
    M, N = x.shape
    q = Eight(M, N, block_rows) if out is None else out
    B.lstm_quantize_fp8(M, N, TYPE[x.dtype], block_rows, x.data_ptr(), x.stride(0), q.codes.data_ptr(), q.codes.stride(0), q.scale.data_ptr(),
                        q.scale.stride(0), _stream())
    return q


def product(a, w, out, bias=None, ws=None):
    """out [a.rows, w.rows] = a w^T + bias"""
    ws = _workspace(B.lstm_matmul_fp8_workspace_bytes(a.rows, w.rows, a.cols)) if ws is None else ws
    B.lstm_matmul_fp8(a.rows, w.rows, a.cols, a.codes.data_ptr(), a.codes.stride(0), a.scale.data_ptr(), a.scale.stride(0),
                      w.codes.data_ptr(), w.codes.stride(0), w.scale.data_ptr(), w.scale.stride(0), w.block_rows, _ptr(bias), TYPE[out.dtype],
                      out.data_ptr(), out.stride(0), ws.data_ptr(), ws.numel(), _stream())
    return out


_held = {}      # one workspace for each stream, as large as any call on it has asked for: calls on a stream follow each other


def _workspace(nbytes):
    """For calls that run now.  What is recorded needs one of its own: this one may be given back for a larger one, and a
    graph may be replayed on another stream."""
    ws = _held.get(_stream())
    if ws is None or ws.numel() < nbytes:
        ws = _held[_stream()] = torch.empty(max(nbytes, 1 << 20), dtype=torch.uint8, device="cuda")
    return ws


def norm(x, residual, weight, y8, sums=None, rstd=None):
    M, N = x.shape
    B.lstm_rmsnorm_forward(M, N, TYPE[x.dtype], x.data_ptr(), x.stride(0), _ptr(residual), N, weight.data_ptr(), EPS, _ptr(sums), N, None, N,
                           y8.codes.data_ptr(), y8.codes.stride(0), y8.scale.data_ptr(), y8.scale.stride(0), _ptr(rstd), _stream())


def norm_gradient(sums, weight, rstd, dy, dsum):
    M, N = sums.shape
    dx, dw = torch.empty_like(sums), torch.empty_like(weight)
    ws = _workspace(B.lstm_rmsnorm_workspace_bytes(M, N))
    B.lstm_rmsnorm_backward(M, N, TYPE[sums.dtype], sums.data_ptr(), N, weight.data_ptr(), rstd.data_ptr(), dy.data_ptr(), N, _ptr(dsum), N,
                            dx.data_ptr(), N, dw.data_ptr(), ws.data_ptr(), ws.numel(), _stream())
    return dx, dw


def scan(P, lengths, c0, h, cT, states=None, ws=None):
    T, batch, H = h.shape
    ws = _workspace(B.lstm_scan_workspace_bytes(T, batch, H)) if ws is None else ws
    B.lstm_scan_forward(T, batch, H, TYPE[P.dtype], False, P.data_ptr(), P.stride(0), P.stride(1), _ptr(lengths), _ptr(c0), h.data_ptr(),
                        h.stride(0), h.stride(1), _ptr(cT), _ptr(states), ws.data_ptr(), ws.numel(), _stream())


def scan_gradient(P, states, dh):
    T, batch, H = dh.shape
    dP = torch.empty_like(P)
    ws = _workspace(B.lstm_scan_workspace_bytes(T, batch, H))
    B.lstm_scan_backward(T, batch, H, TYPE[P.dtype], False, P.data_ptr(), P.stride(0), P.stride(1), None, states.data_ptr(), dh.data_ptr(),
                         dh.stride(0), dh.stride(1), None, dP.data_ptr(), dP.stride(0), dP.stride(1), None, ws.data_ptr(), ws.numel(), _stream())
    return dP


class RecurrentLm:
    def __init__(self, words, units, blocks, seed=0):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)

        def normal(*shape, scale):
            return torch.randn(shape, generator=gen, device="cuda") * scale

        self.words, self.units, self.blocks = words, units, blocks
        p = self.params = {"embedding": normal(words, units, scale=1.0), "norm": torch.ones(units, device="cuda"),
                           "vocabulary": normal(words, units, scale=units ** -0.5)}
        for k in range(blocks):
            b = torch.zeros(4 * units, device="cuda")
            b[:units] = torch.linspace(0, 4, units, device="cuda")      # forget gates that remember from two steps to some fifty
            p.update({f"norm{k}": torch.ones(units, device="cuda"), f"in{k}": normal(4 * units, units, scale=units ** -0.5), f"bias{k}": b,
                      f"out{k}": normal(units, units, scale=units ** -0.5)})
        self.lay_out()

    def lay_out(self):
        """The matrices as the products read them; again after every change of the parameters."""
        self.eight = {k: quantize(v, 128) for k, v in self.params.items() if k == "vocabulary" or k.startswith(("in", "out"))}

    def forward(self, tokens, lengths=None, state=None, keep=None, last_only=False):
        """tokens [T, batch] -> logits (of every step, or of each sequence's last one), new states [blocks, batch, units].
        keep: a list that receives what the gradient needs."""
        (T, batch), H, p = tokens.shape, self.units, self.params
        M = T * batch
        x, residual = p["embedding"][tokens.reshape(-1)].to(torch.bfloat16), None
        new_state = torch.empty((self.blocks, batch, H), device="cuda")
        for k in range(self.blocks):
            y8, sums, rstd = Eight(M, H), torch.empty_like(x), torch.empty(M, device="cuda")
            norm(x, residual, p[f"norm{k}"], y8, sums, rstd)
            P = torch.empty((T, batch, 4 * H), dtype=torch.bfloat16, device="cuda")
            product(y8, self.eight[f"in{k}"], P.view(M, 4 * H), p[f"bias{k}"])
            h = torch.empty((T, batch, H), dtype=torch.bfloat16, device="cuda")
            states = None if keep is None else torch.empty((-(-T // B.LSTM_SCAN_STEPS), batch, H), device="cuda")
            scan(P, lengths, None if state is None else state[k], h, new_state[k], states)
            h8 = quantize(h.view(M, H))
            x, residual = sums, product(h8, self.eight[f"out{k}"], torch.empty_like(x))
            if keep is not None:
                keep.append((sums, rstd, P, states, h))
        if last_only:
            at = torch.full((batch,), T - 1, device="cuda") if lengths is None else (lengths.long() - 1).clamp(min=0)
            rows = at * batch + torch.arange(batch, device="cuda")
            x, residual, M = x[rows], residual[rows], batch
        y8, sums, rstd = Eight(M, H), torch.empty_like(x), torch.empty(M, device="cuda")
        norm(x, residual, p["norm"], y8, sums, rstd)
        if keep is not None:
            keep.append((sums, rstd))
        return product(y8, self.eight["vocabulary"], torch.empty((M, self.words), device="cuda")), new_state

    def gradient(self, tokens, targets):
        """Mean cross-entropy of `targets` [T, batch] and its gradient by every parameter."""
        keep, p, (T, batch), H = [], self.params, tokens.shape, self.units
        M, grad = T * batch, {}
        logits, _ = self.forward(tokens, keep=keep)
        log_p = torch.log_softmax(logits, 1)
        right = targets.reshape(-1, 1)
        loss = -log_p.gather(1, right).mean()
        dlogits = log_p.exp_()
        dlogits.scatter_add_(1, right, torch.full_like(right, -1, dtype=torch.float32))
        dlogits /= M

        def through(name, d, inputs, dtype):
            """dW into `grad`, and the gradient of the inputs [M, columns of W]"""
            w = self.eight[name]
            grad[name] = product(quantize(d.t().contiguous()), quantize(inputs.t().contiguous()), torch.empty((w.rows, w.cols), device="cuda"))
            return product(quantize(d.contiguous()), w.transposed(), torch.empty((M, w.cols), dtype=dtype, device="cuda"))

        sums, rstd = keep.pop()
        normed = (sums * rstd[:, None] * p["norm"]).to(torch.bfloat16)
        dy = through("vocabulary", dlogits, normed, torch.bfloat16)
        dx, grad["norm"] = norm_gradient(sums, p["norm"], rstd, dy, None)
        for k in reversed(range(self.blocks)):
            sums, rstd, P, states, h = keep.pop()
            dh = through(f"out{k}", dx, h.view(M, H), torch.bfloat16)
            dP = scan_gradient(P, states, dh.view(T, batch, H)).view(M, 4 * H)
            grad[f"bias{k}"] = dP.float().sum(0)
            normed = (sums * rstd[:, None] * p[f"norm{k}"]).to(torch.bfloat16)
            dy = through(f"in{k}", dP, normed, torch.bfloat16)
            dx, grad[f"norm{k}"] = norm_gradient(sums, p[f"norm{k}"], rstd, dy, dx)
        grad["embedding"] = torch.zeros_like(p["embedding"]).index_add_(0, tokens.reshape(-1), dx.float())
        return loss, grad


class Writer:
    """Draws token after token of a batch of sequences.  A step's launches are recorded once into a graph."""

    def __init__(self, model, token, state, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
        batch, H = token.numel(), model.units
        self.model, self.token, self.state = model, token.to(torch.int32).clone(), state.clone()
        self.u = torch.empty(batch, device="cuda")
        full = lambda v, dtype: torch.full((batch,), v, dtype=dtype, device="cuda")  # noqa: E731
        self.settings = (full(temperature, torch.float32), full(top_k, torch.int32), full(top_p, torch.float32), full(min_p, torch.float32))
        bf16 = lambda *shape: torch.empty(shape, dtype=torch.bfloat16, device="cuda")  # noqa: E731
        self.embedding = model.params["embedding"].to(torch.bfloat16)
        self.x, self.P, self.h, self.r, self.sums = bf16(batch, H), bf16(1, batch, 4 * H), bf16(1, batch, H), bf16(batch, H), bf16(2, batch, H)
        self.y8, self.h8 = Eight(batch, H), Eight(batch, H)
        self.logits = torch.empty((batch, model.words), device="cuda")
        self.prob, self.kept = torch.empty(batch, device="cuda"), torch.empty(batch, dtype=torch.int32, device="cuda")
        need = [B.lstm_scan_workspace_bytes(1, batch, H), B.lstm_sample_workspace_bytes(batch, model.words)]
        need += [B.lstm_matmul_fp8_workspace_bytes(batch, n, H) for n in (4 * H, H, model.words)]
        self.ws = torch.empty(max(need), dtype=torch.uint8, device="cuda")      # as long as the graph that holds its address
        self.graph = None

    def step(self):
        m, p, batch, H = self.model, self.model.params, self.token.numel(), self.model.units
        torch.index_select(self.embedding, 0, self.token, out=self.x)
        x, residual = self.x, None
        for k in range(m.blocks):
            sums = self.sums[k % 2]
            norm(x, residual, p[f"norm{k}"], self.y8, sums)
            product(self.y8, m.eight[f"in{k}"], self.P.view(batch, 4 * H), p[f"bias{k}"], ws=self.ws)
            scan(self.P, None, self.state[k], self.h, self.state[k], ws=self.ws)        # one step may write its state in place
            quantize(self.h.view(batch, H), out=self.h8)
            x, residual = sums, product(self.h8, m.eight[f"out{k}"], self.r, ws=self.ws)
        norm(x, residual, p["norm"], self.y8)
        product(self.y8, m.eight["vocabulary"], self.logits, ws=self.ws)
        B.lstm_sample(batch, m.words, B.LSTM_F32, self.logits.data_ptr(), m.words, None, 0, *(s.data_ptr() for s in self.settings),
                      self.u.data_ptr(), self.token.data_ptr(), self.prob.data_ptr(), self.kept.data_ptr(), self.ws.data_ptr(), self.ws.numel(),
                      _stream())

    def record(self):
        """Records a step.  Two are run in front of it, on the stream that records and on copies of what they change."""
        token, state = self.token.clone(), self.state.clone()
        self.u.fill_(0.5)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            for _ in range(2):
                self.step()
            self.graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(self.graph, stream=side):
                self.step()
        torch.cuda.current_stream().wait_stream(side)
        self.token.copy_(token)
        self.state.copy_(state)

    def write(self, u):
        """u [steps, batch] uniform numbers -> tokens [steps, batch]"""
        out = torch.empty(u.shape, dtype=torch.int32, device="cuda")
        for i in range(u.shape[0]):
            self.u.copy_(u[i])
            if self.graph is not None:
                self.graph.replay()
            else:
                self.step()
            out[i] = self.token
        return out


def train(model, tokens, steps, rate):
    """`steps` steps of Adam on one batch tokens [T + 1, batch]; the losses."""
    moments = {k: (torch.zeros_like(v), torch.zeros_like(v)) for k, v in model.params.items()}
    losses = []
    for n in range(1, steps + 1):
        loss, grad = model.gradient(tokens[:-1], tokens[1:])
        for k, v in model.params.items():
            m1, m2 = moments[k]
            m1.mul_(0.9).add_(grad[k], alpha=0.1)
            m2.mul_(0.99).addcmul_(grad[k], grad[k], value=0.01)
            v.addcdiv_(m1, (m2 / (1 - 0.99 ** n)).sqrt_().add_(1e-8), value=-rate / (1 - 0.9 ** n))
        model.lay_out()
        losses.append(float(loss))
    return losses


def main():
    a = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    a.add_argument("--words", type=int, default=10000)
    a.add_argument("--units", type=int, default=1500)
    a.add_argument("--blocks", type=int, default=2)
    a.add_argument("--batch", type=int, default=4)
    a.add_argument("--prompt", type=int, default=64, help="tokens of the longest prompt")
    a.add_argument("--generate", type=int, default=64)
    a.add_argument("--train", type=int, default=0, help="steps on one synthetic batch first")
    a = a.parse_args()
    model = RecurrentLm(a.words, a.units, a.blocks)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    # text in which a word decides the next one most of the time
    follows = torch.randperm(a.words, generator=gen, device="cuda")
    tokens = [torch.randint(0, a.words, (a.batch,), generator=gen, device="cuda")]
    for _ in range(a.prompt):
        new = torch.randint(0, a.words, (a.batch,), generator=gen, device="cuda")
        tokens.append(torch.where(torch.rand(a.batch, generator=gen, device="cuda") < 0.9, follows[tokens[-1]], new))
    tokens = torch.stack(tokens)
    if a.train:
        losses = train(model, tokens, a.train, 2e-3)
        print(f"loss {losses[0]:.3f} -> {losses[-1]:.3f} in {a.train} steps")
    lengths = torch.randint(a.prompt // 2, a.prompt + 1, (a.batch,), generator=gen, device="cuda", dtype=torch.int32)
    logits, state = model.forward(tokens[:a.prompt], lengths, last_only=True)
    writer = Writer(model, logits.argmax(1), state, temperature=0.8, top_k=50, top_p=0.95)
    writer.record()
    u = torch.rand((a.generate, a.batch), generator=gen, device="cuda")
    writer.write(u[:2])
    torch.cuda.synchronize()
    start = time.perf_counter()
    out = writer.write(u[2:])
    torch.cuda.synchronize()
    seconds = time.perf_counter() - start
    print(f"{out.numel()} tokens, {1e6 * seconds / max(1, out.shape[0]):.1f} us a step of {a.batch} sequences")
    print("first sequence:", " ".join(str(int(t)) for t in out[:16, 0]))


if __name__ == "__main__":
    main()
