"""Cases of the gated delta rule on the device, against the oracle.

Tolerances.  A step with a key of length 1 and beta in [0, 2] does not lengthen a column of S, and does not lengthen what a rounding
left in one.  What a step adds is rounded in sums over key_dim terms and over up to three times LSTM_DELTA_STEPS terms of the products
inside a block, each off by at most half a step u of fp32 relative to values no larger than the largest column; the roundings of T steps
are independent, so they add like the root of their number.  Eight times that: 8 u sqrt((key_dim + 192) T) times the largest column.
Gradients sum over value_dim too and go through the states twice: 16 u sqrt((key_dim + value_dim + 192) T) times the largest gradient
of the sequence and head.  dbeta and dg of a step are inner products, of two rows of value_dim and of two states: rounding each
of n terms to within u of itself moves their sum by up to u times the sum of the magnitudes, however small the sum comes out, so theirs is relative
to the largest product of the rows' lengths and the largest sum of magnitudes.  Results in bf16: half a step of the value besides."""
import numpy as np

from oracle import lm_ops as O
from paper_1901_10997_amd import binding as B
from tests.lm_ops_util import DTYPE, HALF, U32, Buf, close, dev, ptr, rounded, workspace


def make(seed, T, batch, heads, key_heads, Dk, Dv, name, decay="mixed", beta="sigmoid", state=True, lengths=None):
    r = np.random.default_rng(seed)

    def unit(x):        # queries and keys that share a mean, of length 1 before they are rounded
        x = x / (1 + np.exp(-x)) if Dk > 1 else x
        return x / np.maximum(np.linalg.norm(x, axis=-1, keepdims=True), 1e-3)

    c = dict(T=T, batch=batch, heads=heads, key_heads=key_heads, Dk=Dk, Dv=Dv, name=name, scale=Dk ** -0.5, lengths=lengths)
    c["q"] = rounded(unit(r.normal(size=(T, batch, key_heads, Dk))).reshape(T, batch, key_heads * Dk), name)
    c["k"] = rounded(unit(r.normal(size=(T, batch, key_heads, Dk))).reshape(T, batch, key_heads * Dk), name)
    c["v"] = rounded(r.normal(size=(T, batch, heads * Dv)), name)
    g = -np.exp(r.uniform(np.log(1e-3), 0, size=heads)) * np.log1p(np.exp(r.normal(size=(T, batch, heads))))
    if decay == "strong":       # down to nothing from one step to the next, and now and then all at once
        g = g * 40
        g[r.uniform(size=g.shape) < 0.1] = -np.inf
        g[r.uniform(size=g.shape) < 0.1] = -3e38
    c["g"] = None if decay is None else np.float32(g).astype(np.float64)
    b = {"sigmoid": 1 / (1 + np.exp(-r.normal(size=(T, batch, heads)))), "edges": r.choice([0.0, 1.0, 2.0, 0.5], size=(T, batch, heads))}[beta]
    c["beta"] = np.float32(b).astype(np.float64)
    c["S0"] = np.float32(r.normal(size=(batch, heads, Dk, Dv)) * 0.3).astype(np.float64) if state else None
    c["dO"] = rounded(r.normal(size=(T, batch, heads * Dv)), name)
    c["dST"] = np.float32(r.normal(size=(batch, heads, Dk, Dv)) * 0.3).astype(np.float64)
    return c


def oracle_args(c):
    return (c["q"], c["k"], c["v"], c["g"], c["beta"], c["heads"], c["key_heads"], c["scale"])


def oracle_forward(c):
    return O.delta_forward(*oracle_args(c), lengths=c["lengths"], S0=c["S0"])


def buffers(c, **layout):
    """Inputs on the device: rows of [T, batch], in the given layout."""
    s = {n: Buf(c[n].shape, c["name"], data=c[n], **layout) for n in ("q", "k", "v", "dO")}
    s["beta"] = Buf(c["beta"].shape, "f32", data=c["beta"], **layout)
    s["g"] = None if c["g"] is None else Buf(c["g"].shape, "f32", data=c["g"], **layout)
    s["lengths"] = None if c["lengths"] is None else dev(np.array(c["lengths"], np.int32))
    s["S0"] = None if c["S0"] is None else dev(c["S0"].astype(np.float32))
    s["dST"] = None if c["dST"] is None else dev(c["dST"].astype(np.float32))
    return s


def rows(b):
    return (None, 0, 0) if b is None else (b.ptr, *b.strides)


def inputs_of(c, s):
    sizes = (c["T"], c["batch"], c["heads"], c["key_heads"], c["Dk"], c["Dv"])
    return (*sizes, DTYPE[c["name"]], *rows(s["q"]), *rows(s["k"]), *rows(s["v"]), *rows(s["g"]), *rows(s["beta"]), ptr(s["lengths"]), c["scale"])


def forward(c, s, states=False, ST=None, stream=None, **layout):
    """o (a Buf), the final state and, where asked for, the states that the gradient needs."""
    import torch
    shape = (c["batch"], c["heads"], c["Dk"], c["Dv"])
    o = Buf((c["T"], c["batch"], c["heads"] * c["Dv"]), c["name"], **layout)
    ST = torch.full(shape, 5.0, device="cuda:0") if ST is None else ST
    kept = torch.full((-(-c["T"] // B.LSTM_DELTA_STEPS), *shape), -777.0, device="cuda:0") if states else None
    ws = workspace(B.lstm_delta_workspace_bytes(*inputs_of(c, s)[:6]))
    B.lstm_delta_forward(*inputs_of(c, s), ptr(s["S0"]), *rows(o), ptr(ST), ptr(kept), ptr(ws), ws.numel(), stream)
    return o, ST, kept


def backward(c, s, kept, dS0=None, stream=None, **layout):
    import torch
    T, batch = c["T"], c["batch"]
    keys = (T, batch, c["key_heads"] * c["Dk"])
    out = {"dq": Buf(keys, c["name"], **layout), "dk": Buf(keys, c["name"], **layout),
           "dv": Buf((T, batch, c["heads"] * c["Dv"]), c["name"], **layout), "dg": None if c["g"] is None else Buf(c["g"].shape, "f32", **layout),
           "dbeta": Buf(c["beta"].shape, "f32", **layout)}
    dS0 = torch.full((batch, c["heads"], c["Dk"], c["Dv"]), 5.0, device="cuda:0") if dS0 is None else dS0
    ws = workspace(B.lstm_delta_workspace_bytes(*inputs_of(c, s)[:6], True))
    B.lstm_delta_backward(*inputs_of(c, s), ptr(kept), *rows(s["dO"]), ptr(s["dST"]), *rows(out["dq"]), *rows(out["dk"]), *rows(out["dv"]),
                          *rows(out["dg"]), *rows(out["dbeta"]), ptr(dS0), ptr(ws), ws.numel(), stream)
    return out, dS0


def host(t):
    return t.double().cpu().numpy()


def check_forward(c, o, ST, kept=None):
    want_o, want_S, front = oracle_forward(c)
    T, batch, H, Dv = c["T"], c["batch"], c["heads"], c["Dv"]
    steps = 8 * U32 * np.sqrt((c["Dk"] + 192) * max(T, 1))
    every = np.concatenate((front, want_S[None]))
    largest = np.sqrt((every ** 2).sum(3)).max(axis=(0, 3)) + (abs(c["v"].reshape(T, batch, H, Dv)).max(axis=(0, 3)) if T else 0)    # [batch, heads]
    q = np.repeat(c["q"].reshape(T, batch, c["key_heads"], c["Dk"]), H // c["key_heads"], axis=2)
    found = c["scale"] * np.sqrt((q ** 2).sum(3))[..., None] * largest[None, :, :, None]
    tol = steps * np.broadcast_to(found, (T, batch, H, Dv)).reshape(T, batch, -1) + HALF[c["name"]] * abs(want_o)
    close(o.get() if hasattr(o, "get") else host(o), want_o, tol, "o")
    close(host(ST), want_S, steps * largest[:, :, None, None], "ST")
    if kept is not None:
        n = np.full(batch, T) if c["lengths"] is None else np.clip(c["lengths"], 0, T)
        for i in range(kept.shape[0]):
            for b in range(batch):
                if 64 * i < n[b]:
                    close(host(kept[i, b]), front[64 * i, b], steps * largest[b, :, None, None], "states")
                else:
                    assert bool((kept[i, b] == -777.0).all())


def check_backward(c, out, dS0):
    _, _, front = oracle_forward(c)
    T, batch, H, HK = c["T"], c["batch"], c["heads"], c["key_heads"]
    sizes = {}
    want = dict(zip(("dq", "dk", "dv", "dg", "dbeta", "dS0"), O.delta_backward(*oracle_args(c), front, c["dO"], c["lengths"], c["dST"], sizes)))
    steps = 16 * U32 * np.sqrt((c["Dk"] + c["Dv"] + 192) * max(T, 1))
    for name, of in (("dq", HK), ("dk", HK), ("dv", H), ("dg", H), ("dbeta", H)):
        if out[name] is None:
            continue
        w = want[name]
        largest = abs(sizes.get(name, w).reshape(T, batch, of, -1)).max(axis=(0, 3), initial=0.0)
        tol = steps * np.broadcast_to(largest[None, :, :, None], (T, batch, of, w.size // max(1, T * batch * of))).reshape(w.shape)
        close(out[name].get(), w, tol + (HALF[c["name"]] * abs(w) if name in ("dq", "dk", "dv") else 0), name)
    largest = abs(want["dS0"]).max(axis=(2, 3), keepdims=True)
    close(host(dS0), want["dS0"], steps * np.maximum(largest, abs(c["dST"]).max() if c["dST"] is not None else 0), "dS0")
