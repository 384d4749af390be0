"""Gated delta rule and its gradient against the oracle: sizes on both sides of every tile and block, layouts, lengths, decays that forget
all, shared heads, states in place, single steps, graphs and streams.  How the tolerances come about stands in delta_util.py."""
import numpy as np
import pytest

from paper_1901_10997_amd import binding as B
from tests import delta_util as D
from tests.lm_ops_util import U32, dev, ptr, workspace

pytestmark = pytest.mark.gpu

# T, batch, heads, key_heads, key_dim, value_dim
SHAPES = [
    (1, 1, 1, 1, 1, 1), (1, 3, 4, 2, 125, 125), (2, 2, 2, 1, 64, 33), (8, 1, 2, 2, 128, 130), (1, 2, 1, 1, 256, 31), (5, 1, 3, 3, 129, 16),
    (9, 1, 1, 1, 16, 16), (63, 2, 2, 2, 5, 17), (64, 1, 4, 2, 64, 64), (65, 2, 2, 1, 65, 33), (127, 1, 2, 2, 100, 100), (130, 2, 4, 1, 128, 48),
    (200, 1, 2, 2, 192, 20), (70, 1, 2, 1, 256, 40), (193, 1, 1, 1, 1, 3),
]
IDS = ["x".join(map(str, s)) for s in SHAPES]


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=IDS)
def test_forward(shape, name):
    c = D.make(1, *shape, name)
    D.check_forward(c, *D.forward(c, D.buffers(c), states=True))


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=IDS)
def test_backward(shape, name):
    c = D.make(2, *shape, name)
    s = D.buffers(c)
    _, _, kept = D.forward(c, s, states=True)
    D.check_backward(c, *D.backward(c, s, kept))


@pytest.mark.parametrize("decay,beta,state", [(None, "sigmoid", False), ("strong", "edges", True), ("mixed", "edges", False), (None, "edges", True)])
@pytest.mark.parametrize("T", [7, 150])
@pytest.mark.parametrize("name", ["f32", "bf16"])
def test_gates(name, T, decay, beta, state):
    c = D.make(3, T, 2, 4, 2, 48, 40, name, decay=decay, beta=beta, state=state)
    s = D.buffers(c)
    o, ST, kept = D.forward(c, s, states=True)
    D.check_forward(c, o, ST, kept)
    D.check_backward(c, *D.backward(c, s, kept))


@pytest.mark.parametrize("layout", [dict(pad=3, off=1), dict(pad=8, off=0, order=[1, 0]), dict(pad=1, off=5, order=[1, 0])], ids=["odd", "batch", "odd_batch"])
@pytest.mark.parametrize("T", [6, 140])
@pytest.mark.parametrize("name", ["f32", "bf16"])
def test_layouts_and_lengths(name, T, layout):
    """Rows anywhere, sequences of every length (none, one, all, and out of range), NaN behind the ends."""
    c = D.make(4, T, 6, 2, 1, 36, 50, name, lengths=[T, 0, 1, T + 100, -5, T - 3])
    n = np.clip(c["lengths"], 0, T)
    s = D.buffers(c, **layout)
    for key in ("q", "k", "v", "g", "beta", "dO"):
        for b in range(6):
            s[key].t[n[b]:, b] = float("nan")
    o, ST, kept = D.forward(c, s, states=True, **layout)
    D.check_forward(c, o, ST, kept)
    D.check_backward(c, *D.backward(c, s, kept, **layout))


@pytest.mark.parametrize("T", [1, 4, 100])
def test_states_in_place(T):
    c = D.make(5, T, 2, 2, 2, 64, 70, "f32")
    s = D.buffers(c)
    _, ST, kept = D.forward(c, s, states=True, ST=s["S0"])
    assert ST is s["S0"]
    _, want, _ = D.oracle_forward(c)
    assert abs(D.host(ST) - want).max() <= 8 * U32 * np.sqrt(256 * T) * (abs(want).max() * 8 + 4)
    _, dS0 = D.backward(c, s, kept, dS0=s["dST"])
    fresh = D.buffers(c)
    _, want = D.backward(c, fresh, kept)
    assert bool((dS0 == want).all())


def test_no_state_wanted_and_none_given():
    c = D.make(6, 80, 1, 2, 2, 30, 20, "bf16", state=False)
    c["dST"] = None
    s = D.buffers(c)
    _, _, kept = D.forward(c, s, states=True)
    out, dS0 = D.backward(c, s, kept)
    D.check_backward(c, out, dS0)
    o = D.Buf(c["v"].shape, "bf16")
    ws = workspace(B.lstm_delta_workspace_bytes(*D.inputs_of(c, s)[:6]))
    B.lstm_delta_forward(*D.inputs_of(c, s), None, *D.rows(o), None, None, ptr(ws), ws.numel())
    want, _, _ = D.forward(c, s)
    assert np.array_equal(o.get(), want.get())


def test_nothing_to_walk():
    """No steps move the state; no sequences do nothing."""
    import torch
    c = D.make(7, 20, 2, 2, 2, 8, 8, "f32")
    s = D.buffers(c)
    ST, dS0, ws = torch.zeros_like(s["S0"]), torch.zeros_like(s["S0"]), workspace(256)
    sizes = list(D.inputs_of(c, s))
    none = [0] + sizes[1:]
    B.lstm_delta_forward(*none, ptr(s["S0"]), None, 0, 0, ptr(ST), None, ptr(ws), 256)
    B.lstm_delta_backward(*none, None, None, 0, 0, ptr(s["dST"]), *[None, 0, 0] * 5, ptr(dS0), ptr(ws), 256)
    torch.cuda.synchronize()
    assert bool((ST == s["S0"]).all()) and bool((dS0 == s["dST"]).all())
    sizes[1] = 0
    B.lstm_delta_forward(*sizes, ptr(s["S0"]), None, 0, 0, ptr(dS0), None, ptr(ws), 256)
    torch.cuda.synchronize()
    assert bool((dS0 == s["dST"]).all())


@pytest.mark.parametrize("name", ["f32", "bf16"])
def test_steps_follow_a_prompt(name):
    """A prompt in blocks, then token after token in place: what the oracle has of the whole sequence."""
    c = D.make(8, 75, 3, 4, 2, 64, 48, name)
    s = D.buffers(c)
    head = dict(c, T=70)
    state = s["S0"]
    o = D.Buf(c["v"].shape, name)
    ws = workspace(max(B.lstm_delta_workspace_bytes(70, 3, 4, 2, 64, 48), B.lstm_delta_workspace_bytes(1, 3, 4, 2, 64, 48)))
    args = list(D.inputs_of(head, s))
    B.lstm_delta_forward(*args, ptr(state), *D.rows(o), ptr(state), None, ptr(ws), ws.numel())
    size = o.t.element_size()
    for t in range(70, 75):
        args[0] = 1
        for at, b in ((7, s["q"]), (10, s["k"]), (13, s["v"]), (16, s["g"]), (19, s["beta"])):
            args[at] = b.ptr + t * b.strides[0] * b.t.element_size()
        B.lstm_delta_forward(*args, ptr(state), o.ptr + t * o.strides[0] * size, *o.strides, ptr(state), None, ptr(ws), ws.numel())
    D.check_forward(c, o, state)


def test_one_sequence_does_not_see_another():
    """A NaN, an infinity or an enormous value of one sequence and head leaves the bits of all others."""
    c = D.make(9, 90, 3, 4, 2, 32, 24, "f32")
    s = D.buffers(c)
    clean = [x.clone() for x in (D.forward(c, s)[0].t, D.forward(c, s)[1])]
    s["v"].t[20, 1, 24 * 3 + 5] = float("nan")
    s["beta"].t[70, 1, 2] = float("inf")
    s["g"].t[3, 1, 0] = float("nan")
    o, ST, _ = D.forward(c, s)
    for b in (0, 2):
        assert bool((o.t[:, b] == clean[0][:, b]).all()) and bool((ST[b] == clean[1][b]).all())
    assert bool((o.t[:, 1, 24:48] == clean[0][:, 1, 24:48]).all())        # head 1 of the same sequence
    assert bool(o.t[20:, 1, 24 * 3 + 5].isnan().all()) and bool((o.t[:, 1, 24 * 3:24 * 3 + 5] == clean[0][:, 1, 24 * 3:24 * 3 + 5]).all())
    assert bool(ST[1, 0].isnan().all())


@pytest.mark.parametrize("T", [3, 130])
def test_same_bits_again_on_streams_and_in_a_graph(T):
    import torch
    c = D.make(10, T, 2, 4, 2, 64, 64, "bf16")
    s = D.buffers(c)
    o, ST, kept = D.forward(c, s, states=True)
    out, dS0 = D.backward(c, s, kept)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        o2, ST2, kept2 = D.forward(c, s, states=True, stream=side.cuda_stream)
        out2, dS02 = D.backward(c, s, kept2, stream=side.cuda_stream)
    side.synchronize()
    assert bool((o2.t == o.t).all()) and bool((ST2 == ST).all()) and bool((dS02 == dS0).all())
    assert all(bool((out2[k].t == out[k].t).all()) for k in out)
    # recorded: the same buffers with other values in them between the replays
    sizes = D.inputs_of(c, s)[:6]
    ws, ws_back = workspace(B.lstm_delta_workspace_bytes(*sizes)), workspace(B.lstm_delta_workspace_bytes(*sizes, True))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        st = torch.cuda.current_stream().cuda_stream
        B.lstm_delta_forward(*D.inputs_of(c, s), ptr(s["S0"]), *D.rows(o2), ptr(ST2), ptr(kept2), ptr(ws), ws.numel(), st)
        B.lstm_delta_backward(*D.inputs_of(c, s), ptr(kept2), *D.rows(s["dO"]), ptr(s["dST"]), *D.rows(out2["dq"]), *D.rows(out2["dk"]), *D.rows(out2["dv"]),
                              *D.rows(out2["dg"]), *D.rows(out2["dbeta"]), ptr(dS02), ptr(ws_back), ws_back.numel(), st)
    for turn in range(3):
        s["v"].t.mul_(1.5)
        s["dO"].t.neg_()
        graph.replay()
        torch.cuda.synchronize()
        o3, ST3, kept3 = D.forward(c, s, states=True)
        out3, dS03 = D.backward(c, s, kept3)
        torch.cuda.synchronize()
        assert bool((o2.t == o3.t).all()) and bool((ST2 == ST3).all()) and bool((dS02 == dS03).all())
        assert all(bool((out2[k].t == out3[k].t).all()) for k in out3)


@pytest.mark.parametrize("T", [3, 70])
def test_rows_further_apart_than_32_bits_count(T):
    """Strides whose products with t and b pass 2^32 elements."""
    import torch
    c = D.make(11, T, 2, 2, 1, 16, 20, "bf16")
    near = D.buffers(c)
    o, ST, kept = D.forward(c, near, states=True)
    far, step = dict(near), 2 ** 33 // T // 2 * 2
    store = torch.empty(step * T + 2 ** 10, dtype=torch.bfloat16, device="cuda:0")

    class Far:
        def __init__(self, like, at):
            self.strides = [step, 128]
            self.t = store.as_strided(like.t.shape, self.strides + [1], at)
            self.t.copy_(like.t)
            self.ptr = self.t.data_ptr()

    for i, key in enumerate(("q", "k", "v")):       # 16, 16 and 40 columns at places of their own in rows of 128
        far[key] = Far(near[key], 40 * i)
    o2, ST2, _ = D.forward(c, far)
    assert bool((o2.t == o.t).all()) and bool((ST2 == ST).all())
    out, dS0 = D.backward(c, near, kept)
    out2, dS02 = D.backward(c, far, kept)
    assert bool((dS0 == dS02).all()) and all(bool((out[k].t == out2[k].t).all()) for k in out)
    del store


def test_a_step_too_many_sequences_for_one_round():
    """More workgroups than the device holds at once, several rounds of them."""
    c = D.make(12, 1, 600, 2, 2, 32, 64, "bf16")
    D.check_forward(c, *D.forward(c, D.buffers(c))[:2])


# enough workgroups for two tiles of columns each: one tile and a part of one behind them, an odd one, key columns of both sizes
@pytest.mark.parametrize("T,batch,heads,key_heads,Dk,Dv", [(130, 16, 16, 4, 40, 33), (70, 32, 8, 8, 100, 20), (65, 8, 8, 2, 128, 130), (66, 64, 8, 8, 16, 16)])
@pytest.mark.parametrize("name", ["f32", "bf16"])
def test_many_sequences(name, T, batch, heads, key_heads, Dk, Dv):
    r = np.random.default_rng(13)
    c = D.make(13, T, batch, heads, key_heads, Dk, Dv, name, lengths=[T] + list(r.integers(0, T + 1, batch - 1)))
    s = D.buffers(c)
    o, ST, kept = D.forward(c, s, states=True)
    D.check_forward(c, o, ST, kept)
    D.check_backward(c, *D.backward(c, s, kept))
    plain, ST2, _ = D.forward(c, s)             # the walk that keeps no states
    assert bool((plain.t == o.t).all()) and bool((ST2 == ST).all())


def test_a_walk_does_not_depend_on_its_company():
    """The same sequence alone (one tile to a workgroup) and among many (two): the same bits."""
    c = D.make(14, 130, 40, 8, 4, 64, 48, "bf16")
    many = D.buffers(c)
    o, ST, kept = D.forward(c, many, states=True)
    out, dS0 = D.backward(c, many, kept)
    one = {k: (v[:, 3:4] if k in ("q", "k", "v", "g", "beta", "dO") else v[3:4] if v is not None else None) for k, v in c.items()
           if k in ("q", "k", "v", "g", "beta", "dO", "S0", "dST")}
    alone = dict(c, batch=1, **one)
    s = D.buffers(alone)
    o1, ST1, kept1 = D.forward(alone, s, states=True)
    out1, dS01 = D.backward(alone, s, kept1)
    assert bool((o1.t[:, 0] == o.t[:, 3]).all()) and bool((ST1[0] == ST[3]).all()) and bool((dS01[0] == dS0[3]).all())
    assert all(bool((out1[k].t[:, 0] == out[k].t[:, 3]).all()) for k in out)


def test_keys_of_any_length():
    """Keys are used as they are: short and long ones, whose states stay small, over a few blocks."""
    c = D.make(15, 140, 2, 2, 2, 24, 20, "f32")
    c["k"] = np.float32(c["k"] * 0.3).astype(np.float64)
    c["q"] = np.float32(c["q"] * 50).astype(np.float64)
    s = D.buffers(c)
    o, ST, kept = D.forward(c, s, states=True)
    D.check_forward(c, o, ST, kept)
    D.check_backward(c, *D.backward(c, s, kept))


def test_workspaces_of_their_own():
    """Two calls on two streams at the same time."""
    import torch
    cases = [D.make(16 + i, 200, 2, 4, 2, 64, 64, "bf16") for i in range(2)]
    held = [D.buffers(c) for c in cases]
    want = [D.forward(c, s)[0].t.clone() for c, s in zip(cases, held)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for turn in range(4):
        for c, s, st in zip(cases, held, streams):
            with torch.cuda.stream(st):
                got.append(D.forward(c, s, stream=st.cuda_stream)[0].t)
    torch.cuda.synchronize()
    assert all(bool((g == want[i % 2]).all()) for i, g in enumerate(got))


@pytest.mark.parametrize("T", [8, 60, 150])
def test_growth(T):
    """A gate above 0: with beta = 0 the state only grows, o = scale e^(sum of g) S0'q, up to a sum of 80 in a block."""
    c = D.make(17, T, 2, 2, 1, 40, 24, "f32")
    c["beta"] = np.zeros_like(c["beta"])
    c["g"] = np.full_like(c["g"], 0.5)
    c["g"][64:] = 0.125
    o, ST, _ = D.forward(c, D.buffers(c))
    grown = np.exp(np.cumsum(c["g"], 0))[..., None]                     # [T, batch, heads, 1]
    q = c["q"].reshape(T, 2, 40)
    want = c["scale"] * np.einsum("tbd,bhdv->tbhv", q, c["S0"]) * grown
    # an exponential of up to 47: its argument's rounding 47 u, and that of up to three blocks or of the single steps; sums over 40 terms, relative to their magnitudes
    size = c["scale"] * np.einsum("tbd,bhdv->tbhv", np.abs(q), np.abs(c["S0"])) * grown
    assert (np.abs(D.host(o.t).reshape(T, 2, 2, 24) - want) <= 3 * (47 + 40 + 8) * 2.0 ** -24 * size).all()
    size = np.abs(c["S0"]) * grown[-1][..., None]
    assert (np.abs(D.host(ST) - c["S0"] * grown[-1][..., None]) <= 3 * (47 + 40 + 8) * 2.0 ** -24 * size).all()
