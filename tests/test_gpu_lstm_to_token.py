"""From the stacks of the library to a token: what lstm_forward leaves goes through the norm, the product with the vocabulary and the
draw, one call behind the other on a stream, step by step with the states carried on, against the oracles."""
import numpy as np
import pytest

from lm_ops_util import U32, close, workspace
from oracle import lm_ops as oracle
from oracle import lstm_oracle
from paper_1901_10997_amd import binding as B
from paper_1901_10997_amd import inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,bidirectional,keep", [("f32", False, 0.2), ("f32", True, None), ("bf16", False, None)])
def test_prompt_and_next_words(dtype, bidirectional, keep):
    import torch
    T, batch, D, H, words, steps = 9, 5, 96, 160, 700, 1 if bidirectional else 4
    case = inputs.make_case(inputs.Workload(93, "to_token", 2, bidirectional, D, H, T + steps - 1, batch, dtype, 0.2, keep, "uniform"), k=3)
    model = B.Lstm(2, D, H, bidirectional, B.LSTM_BF16 if dtype == "bf16" else B.LSTM_F32)
    model.set_weights_from(case.weights)
    x = torch.from_numpy(case.x).to("cuda:0").to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    N = model.ndir * H
    rng = np.random.default_rng(11)
    v8, v_scale = oracle.quantize(rng.standard_normal((words, N)).astype(np.float32), 128)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to("cuda:0")  # noqa: E731
    W, Ws, weight = dev(v8), dev(v_scale), dev(np.full(N, 1.5, np.float32))
    u = rng.random((steps, batch)).astype(np.float32)
    ud, k, p = dev(u), dev(np.full(batch, 40, np.int32)), dev(np.full(batch, 0.9, np.float32))
    y8, scale = torch.zeros((batch, N), dtype=torch.uint8, device="cuda:0"), torch.empty((batch, -(-N // 128)), device="cuda:0")
    logits = torch.empty((steps, batch, words), device="cuda:0")
    token, prob, kept = torch.empty((steps, batch), dtype=torch.int32, device="cuda:0"), torch.empty((steps, batch), device="cuda:0"), torch.empty((steps, batch), dtype=torch.int32, device="cuda:0")
    ws, ys, states = workspace(256), [], (None, None)
    codes, scales = [], []
    st = torch.cuda.current_stream().cuda_stream
    for s in range(steps):
        y, *states = model.forward(x[:T] if s == 0 else x[T + s - 1:T + s], *states, stream=st, check=False)
        ys.append(y)
        last = y[-1]
        B.lstm_rmsnorm_forward(batch, N, B.LSTM_F32, last.data_ptr(), N, None, 0, weight.data_ptr(), 1e-5, None, 0, None, 0, y8.data_ptr(), N, scale.data_ptr(),
                               scale.stride(0), None, st)
        B.lstm_matmul_fp8(batch, words, N, y8.data_ptr(), N, scale.data_ptr(), scale.stride(0), W.data_ptr(), N, Ws.data_ptr(), Ws.stride(0), 128, None,
                          B.LSTM_F32, logits[s].data_ptr(), words, ws.data_ptr(), ws.numel(), st)
        B.lstm_sample(batch, words, B.LSTM_F32, logits[s].data_ptr(), words, None, 0, None, k.data_ptr(), p.data_ptr(), None, ud[s].data_ptr(), token[s].data_ptr(),
                      prob[s].data_ptr(), kept[s].data_ptr(), ws.data_ptr(), ws.numel(), st)
        codes.append(y8.clone())
        scales.append(scale.clone())
    torch.cuda.synchronize()
    B.lstm_check(model.handle)
    want_y, *_ = lstm_oracle.forward_case(case)
    got_y = torch.cat(ys).double().cpu().numpy()
    far = np.linalg.norm(got_y - want_y) / np.linalg.norm(want_y)
    assert far <= (2e-2 if dtype == "bf16" else 1e-4)           # the stack's own tolerance
    for s in range(steps):
        last = ys[s][-1].cpu().numpy()
        want, _ = oracle.rmsnorm(last, np.full(N, 1.5), 1e-5)
        a8, a_scale = codes[s].cpu().numpy(), scales[s].cpu().numpy()
        values = oracle.e4m3_decode(a8) * oracle.spread(a_scale.astype(np.float64), 1, batch, N)
        # half a step of e4m3, and half its smallest step, which is 2^-9 of a scale
        close(values, want, 2.0 ** -4 * np.abs(want) * 1.001 + 2.0 ** -10 * oracle.spread(a_scale.astype(np.float64), 1, batch, N) * 1.001)
        want, size = oracle.matmul(a8, a_scale, v8, v_scale, 128)
        got = logits[s].cpu().numpy()
        close(got, want, (128 + N / 128 + 8) * U32 * size)
        for m in range(batch):
            j, q, n = oracle.sample(got[m], u[s, m], top_k=40, top_p=float(np.float32(0.9)))
            assert (int(token[s, m]), int(kept[s, m])) == (j, n)
            assert abs(float(prob[s, m]) - q) <= 2.0 ** -23
    model.close()
