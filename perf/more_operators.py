"""A recurrent language model's memory, its scores and its teacher, as cases that can be timed: the gated delta rule (a
recurrence whose state is a matrix for each head) with its gradient and its form for single tokens, log probabilities of given
tokens with entropy, rank and top alternatives and their gradient, and the distillation loss from a teacher's top logits with
its gradient.  `own` says whether run() makes the library's calls or computes the plain forms: elementary tensor operations in
32 bits (64 where a border or a cancellation decides), rounded once at the end.

listed() names the cases, draw() gives more of the same ranges, prepare() builds what a user's program holds before the call,
run() is one pass, exact() the same outputs from the definitions in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

STEPS = 64             # the delta rule's forward keeps one state for so many steps where a gradient is wanted

# Heads of the widths of the latency profile, speech and language-model batches, utterances and sequences up to documents
HEADS = (1, 32)
HEAD_DIM = (16, 256)
BATCH = (1, 64)
LENGTH = (1, 8192)
MAX_UPDATES = 8192 * 16 * 128 * 128
ROWS = (1, 4096)
VOCABULARY = (256, 131072)
MAX_SCORED = 4096 * 10000
MAX_DISTILLED = 2048 * 32000


def _delta(name, T, B, heads, key_heads, Dk, Dv, dtype, train=False, ragged=False, state=True, decay=True):
    return _named(name, kind="delta", T=T, B=B, heads=heads, key_heads=key_heads, Dk=Dk, Dv=Dv, dtype=dtype, train=train, ragged=ragged,
                  state=state, decay=decay)


def _score(name, M, V, dtype, top=0, masked=False, train=False):
    return _named(name, kind="score", M=M, V=V, dtype=dtype, top=top, masked=masked, train=train)


def _distill(name, M, V, K, dtype, temperature=1.0, rest=True, train=True):
    return _named(name, kind="distill", M=M, V=V, K=K, dtype=dtype, temperature=temperature, rest=rest, train=train)


def _named(name, **c):
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token of one user, 1500 units as twelve heads: latency alone
        _delta("delta_step_b1_12x125", 1, 1, 12, 12, 125, 125, "f32"),
        # one token of each of 64 users, 2048 units, queries and keys shared by two heads: the states' way through memory
        _delta("delta_step_b64_16x128", 1, 64, 16, 8, 128, 128, "bf16"),
        # a document read in one go, one sequence
        _delta("delta_long_b1_t8192", 8192, 1, 16, 16, 128, 128, "bf16"),
        # utterances of different length, 800 units, forward and gradient in fp32
        _delta("delta_speech_b16_t300", 300, 16, 8, 8, 100, 100, "f32", train=True, ragged=True, state=False),
        # a training step's recurrence, 2048 units: forward and gradient
        _delta("delta_train_b8_t1024", 1024, 8, 16, 8, 128, 128, "bf16", train=True),
        # what one user's next word could have been, 10 000 words
        _score("score_1x10000_top5", 1, 10000, "f32", top=5),
        # the tokens of a full batch with their alternatives, each request with a mask of its own
        _score("score_256x32000_top20", 256, 32000, "bf16", top=20, masked=True),
        # likelihood of 20 sequences of 35 words and its gradient by the logits
        _score("score_train_700x10000", 700, 10000, "f32", train=True),
        # the likelihood of a prompt's tokens alone
        _score("score_prompt_4096x10000", 4096, 10000, "bf16"),
        # a language-model batch learns from the 32 likeliest words of a teacher
        _distill("distill_700x10000_k32", 700, 10000, 32, "f32", temperature=2.0),
        # a larger batch and vocabulary, 64 words, the teacher's list taken for the whole of it
        _distill("distill_2048x32000_k64", 2048, 32000, 64, "bf16", rest=False),
        # how far a small model is from its teacher: the loss alone
        _distill("distill_loss_35x2000_k16", 35, 2000, 16, "f32", train=False),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["delta", "delta", "delta", "score", "score", "distill"])
    dtype = rng.choice(["f32", "bf16"])
    if kind == "delta":
        key_heads = _log_int(rng, *HEADS)
        heads = key_heads * rng.choice([n for n in (1, 1, 2, 4) if key_heads * n <= HEADS[1]])
        Dk, Dv = _log_int(rng, *HEAD_DIM), _log_int(rng, *HEAD_DIM)
        if rng.random() < 0.4:
            Dk = Dv = rng.choice([64, 128])
        B = _log_int(rng, *BATCH)
        T = 1 if rng.random() < 0.2 else _log_int(rng, *LENGTH)
        T = max(1, min(T, MAX_UPDATES // (2 if dtype == "f32" else 1) // (B * heads * Dk * Dv)))
        return _delta(None, T, B, heads, key_heads, Dk, Dv, dtype, train=rng.random() < 0.4, ragged=rng.random() < 0.3,
                      state=rng.random() < 0.7, decay=rng.random() < 0.8)
    V = _log_int(rng, *VOCABULARY)
    if kind == "score":
        M = max(1, min(_log_int(rng, *ROWS), MAX_SCORED // (2 if dtype == "f32" else 1) // V))
        train = rng.random() < 0.4
        return _score(None, M, V, dtype, top=0 if train else rng.choice([0, _log_int(rng, 1, 64)]), masked=rng.random() < 0.3, train=train)
    M = max(1, min(_log_int(rng, *ROWS), MAX_DISTILLED // (2 if dtype == "f32" else 1) // V))
    return _distill(None, M, V, _log_int(rng, 1, 128), dtype, temperature=rng.choice([1.0, 2.0, round(rng.uniform(0.5, 4.0), 2)]),
                    rest=rng.random() < 0.6, train=rng.random() < 0.7)


# ---- inputs --------------------------------------------------------------------------------------------------------------

def _type(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _blocks(n, of=STEPS):
    return -(-n // of)


def prepare(case, seed):
    dev = torch.device("cuda:0")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    return {"delta": _prepare_delta, "score": _prepare_score, "distill": _prepare_distill}[case["kind"]](case, gen, dev)


def _prepare_delta(c, gen, dev):
    T, B, H, HK, Dk, Dv, dt = c["T"], c["B"], c["heads"], c["key_heads"], c["Dk"], c["Dv"], _type(c["dtype"])

    def normal(*shape):
        return torch.randn(shape, generator=gen, device=dev)

    def unit(x):        # queries and keys behind a nonlinearity, normed per head: they share a mean
        x = x * torch.sigmoid(x)
        return x / (x.square().sum(-1, keepdim=True) + 1e-6).sqrt()

    # queries, keys and values side by side, as one projection leaves them
    wide = torch.empty((T, B, 2 * HK * Dk + H * Dv), dtype=dt, device=dev)
    q, k, v = wide[:, :, :HK * Dk], wide[:, :, HK * Dk:2 * HK * Dk], wide[:, :, 2 * HK * Dk:]
    q.copy_(unit(normal(T, B, HK, Dk)).view(T, B, HK * Dk))
    k.copy_(unit(normal(T, B, HK, Dk)).view(T, B, HK * Dk))
    v.copy_(normal(T, B, H * Dv))
    # heads that forget within a step or two and heads that keep for a thousand
    rate = torch.exp(torch.rand((H,), generator=gen, device=dev) * math.log(1000.0)) * 1e-3
    s = dict(case=c, q=q, k=k, v=v, beta=torch.sigmoid(normal(T, B, H)), lengths=None, scale=Dk ** -0.5,
             g=-rate * torch.log1p(torch.exp(normal(T, B, H))) if c["decay"] else None,
             S0=normal(B, H, Dk, Dv) * 0.3 if c["state"] else None, ST=torch.empty((B, H, Dk, Dv), device=dev),
             o=torch.empty((T, B, H * Dv), dtype=dt, device=dev))
    if c["ragged"]:
        n = torch.randint(0, T + 1, (B,), generator=gen, device=dev, dtype=torch.int32)
        n[0] = T
        s["lengths"] = n
    if c["train"]:
        s.update(do=normal(T, B, H * Dv).to(dt), dST=normal(B, H, Dk, Dv) * 0.3, dS0=torch.empty((B, H, Dk, Dv), device=dev),
                 states=torch.empty((_blocks(T), B, H, Dk, Dv), device=dev), dq=torch.empty((T, B, HK * Dk), dtype=dt, device=dev),
                 dk=torch.empty((T, B, HK * Dk), dtype=dt, device=dev), dv=torch.empty((T, B, H * Dv), dtype=dt, device=dev),
                 dg=torch.empty((T, B, H), device=dev), dbeta=torch.empty((T, B, H), device=dev))
    return s


def _prepare_logits(M, V, gen, dev):
    """A trained model's logits: most rows have one word far above the rest."""
    logits = torch.randn((M, V), generator=gen, device=dev) * 2.5
    right = torch.randint(0, V, (M, 1), generator=gen, device=dev)
    return logits.scatter_add_(1, right, torch.rand((M, 1), generator=gen, device=dev) * 16), right[:, 0]


def _prepare_score(c, gen, dev):
    M, V, n = c["M"], c["V"], c["top"]
    logits, right = _prepare_logits(M, V, gen, dev)
    other = torch.randint(0, V, (M,), generator=gen, device=dev)
    token = torch.where(torch.rand((M,), generator=gen, device=dev) < 0.7, right, other)
    if M > 8:
        token[torch.rand((M,), generator=gen, device=dev) < 0.05] = -1         # padding
    s = dict(case=c, logits=logits.to(_type(c["dtype"])), token=token.to(torch.int32), allowed=None,
             logprob=torch.empty((M,), device=dev), rank=torch.empty((M,), dtype=torch.int32, device=dev),
             entropy=torch.empty((M,), device=dev), stats=None, top_token=None, top_logprob=None)
    if c["masked"]:     # a grammar or a list of banned words; what is masked holds anything
        s["allowed"] = (torch.rand((M, V), generator=gen, device=dev) < 0.8).to(torch.uint8)
        s["logits"][s["allowed"] == 0] = float("nan")
    if n:
        s.update(top_token=torch.empty((M, n), dtype=torch.int32, device=dev), top_logprob=torch.empty((M, n), device=dev))
    if c["train"]:      # the mean likelihood, and a little entropy to keep
        s.update(stats=torch.empty((M, 4), device=dev), dlogits=torch.empty((M, V), dtype=_type(c["dtype"]), device=dev),
                 dlogprob=torch.full((M,), -1.0 / M, device=dev) * (0.5 + torch.rand((M,), generator=gen, device=dev)),
                 dentropy=torch.full((M,), -0.01 / M, device=dev))
    return s


def _prepare_distill(c, gen, dev):
    M, V, K = c["M"], c["V"], min(c["K"], c["V"])
    logits, _ = _prepare_logits(M, V, gen, dev)
    teacher = torch.randn((M, V), generator=gen, device=dev).add_(logits)
    top_logit, top_token = torch.topk(teacher, K, dim=1)
    lse = torch.logsumexp((teacher / c["temperature"]).double(), 1).float() if c["rest"] else None
    s = dict(case=c, logits=logits.to(_type(c["dtype"])), top_token=top_token.to(torch.int32), top_logit=top_logit.contiguous(), teacher_lse=lse,
             loss=torch.empty((M,), device=dev), stats=None)
    if c["train"]:
        s.update(stats=torch.empty((M, 4), device=dev), dloss=torch.rand((M,), generator=gen, device=dev) / M,
                 dlogits=torch.empty((M, V), dtype=_type(c["dtype"]), device=dev))
    return s


# ---- one pass ------------------------------------------------------------------------------------------------------------

def run(s):
    return (_OWN if own else _PLAIN)[s["case"]["kind"]](s)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _workspace(s, nbytes):
    if "ws" not in s:       # kept from call to call, as a user's program keeps it
        s["ws"] = torch.empty((max(nbytes, 256),), dtype=torch.uint8, device="cuda:0")
    return s["ws"]


def _rows(t):
    """Address and strides of [T, B, ...]; of what is not there, none."""
    return (None, 0, 0) if t is None else (t.data_ptr(), t.stride(0), t.stride(1))


def _own_delta(s):
    from paper_1901_10997_amd import binding as L
    c, ptr = s["case"], _ptr
    sizes = (c["T"], c["B"], c["heads"], c["key_heads"], c["Dk"], c["Dv"])
    if "ws" not in s:
        _workspace(s, L.lstm_delta_workspace_bytes(*sizes, c["train"]))
    ws, stream = s["ws"], torch.cuda.current_stream().cuda_stream
    inputs = (*sizes, L.LSTM_BF16 if c["dtype"] == "bf16" else L.LSTM_F32, *_rows(s["q"]), *_rows(s["k"]), *_rows(s["v"]), *_rows(s["g"]),
              *_rows(s["beta"]), ptr(s["lengths"]), s["scale"])
    L.lstm_delta_forward(*inputs, ptr(s["S0"]), *_rows(s["o"]), ptr(s["ST"]), ptr(s.get("states")), ptr(ws), ws.numel(), stream)
    if not c["train"]:
        return dict(o=s["o"], ST=s["ST"])
    dg = s["dg"] if c["decay"] else None
    L.lstm_delta_backward(*inputs, ptr(s["states"]), *_rows(s["do"]), ptr(s["dST"]), *_rows(s["dq"]), *_rows(s["dk"]), *_rows(s["dv"]),
                          *_rows(dg), *_rows(s["dbeta"]), ptr(s["dS0"]), ptr(ws), ws.numel(), stream)
    return _delta_outputs(s["o"], s["ST"], s["dq"], s["dk"], s["dv"], dg, s["dbeta"], s["dS0"])


def _delta_outputs(o, ST, dq, dk, dv, dg, dbeta, dS0):
    out = dict(o=o, ST=ST, dq=dq, dk=dk, dv=dv, dg=dg, dbeta=dbeta, dS0=dS0)
    return {k: v for k, v in out.items() if v is not None}


def _own_score(s):
    from paper_1901_10997_amd import binding as L
    c, ptr = s["case"], _ptr
    M, V, n = c["M"], c["V"], c["top"]
    if "ws" not in s:
        _workspace(s, L.lstm_logprobs_workspace_bytes(M, V, n))
    ws, stream = s["ws"], torch.cuda.current_stream().cuda_stream
    rows = (M, V, L.LSTM_BF16 if c["dtype"] == "bf16" else L.LSTM_F32, ptr(s["logits"]), V, ptr(s["allowed"]), V, ptr(s["token"]))
    L.lstm_logprobs_forward(*rows, ptr(s["logprob"]), ptr(s["rank"]), ptr(s["entropy"]), ptr(s["stats"]), n, ptr(s["top_token"]),
                            ptr(s["top_logprob"]), ptr(ws), ws.numel(), stream)
    if c["train"]:
        L.lstm_logprobs_backward(*rows, ptr(s["stats"]), ptr(s["dlogprob"]), ptr(s["dentropy"]), ptr(s["dlogits"]), V, stream)
    return _score_outputs(s["logprob"], s["rank"], s["entropy"], s["top_token"], s["top_logprob"], s.get("dlogits"))


def _score_outputs(logprob, rank, entropy, top_token, top_logprob, dlogits):
    """A place for each output, so that None may stand for one without a value."""
    out = dict(logprob=logprob, rank=rank, entropy=entropy)
    if top_logprob is not None:
        out.update(top_token=top_token, top_logprob=top_logprob)
    return out if dlogits is None else dict(out, dlogits=dlogits)


def _own_distill(s):
    from paper_1901_10997_amd import binding as L
    c, ptr = s["case"], _ptr
    M, V, K = c["M"], c["V"], s["top_token"].shape[1]
    if "ws" not in s:
        _workspace(s, L.lstm_distill_workspace_bytes(M, V, K))
    ws, stream = s["ws"], torch.cuda.current_stream().cuda_stream
    rows = (M, V, K, L.LSTM_BF16 if c["dtype"] == "bf16" else L.LSTM_F32, ptr(s["logits"]), V, ptr(s["top_token"]), K, ptr(s["top_logit"]), K,
            ptr(s["teacher_lse"]), c["temperature"])
    L.lstm_distill_forward(*rows, ptr(s["loss"]), ptr(s["stats"]), ptr(ws), ws.numel(), stream)
    if not c["train"]:
        return s["loss"]
    L.lstm_distill_backward(*rows, ptr(s["stats"]), ptr(s["dloss"]), ptr(s["dlogits"]), V, stream)
    return s["loss"], s["dlogits"]


# The plain delta rule goes by blocks of STEPS steps.  With G the running sum of the log decays inside a block, S the state in
# front of it, y = exp(G), e = exp(G_last - G), D_ij = exp(G_i - G_j) for j <= i:
#     R = beta (V - y K S)      U = (I + L)^-1 R,  L_ij = beta_i D_ij k_i.k_j (j < i)
#     O = scale (y Q S + P U),  P_ij = D_ij q_i.k_j (j <= i)         S' = exp(G_last) S + (e K)^T U

def _in_blocks(x, lengths, heads):
    """[T, B, heads * D] as [B, heads, blocks, STEPS, D] in 32 bits, zeros behind the end."""
    T, B = x.shape[:2]
    x = x.float().reshape(T, B, heads, -1)
    if lengths is not None:
        x = torch.where((torch.arange(T, device=x.device)[:, None] < lengths)[:, :, None, None], x, 0.0)
    x = torch.cat((x, x.new_zeros((_blocks(T) * STEPS - T, *x.shape[1:]))))
    return x.permute(1, 2, 0, 3).reshape(B, heads, _blocks(T), STEPS, -1)


def _in_steps(x, T):
    """And back, [T, B, heads * D]."""
    B, heads, n, steps, D = x.shape
    return x.reshape(B, heads, n * steps, D)[:, :, :T].permute(2, 0, 1, 3).reshape(T, B, heads * D)


def _inverse(L):
    """(I + L)^-1 of strictly lower matrices: the diagonal blocks' inverses, of twice the size in each turn."""
    X = torch.eye(STEPS, device=L.device).expand(L.shape).contiguous()
    at = torch.arange(STEPS, device=L.device)
    size = 1
    while size < STEPS:
        low = ((at[:, None] // size == at[None] // size + 1) & (at[:, None] // size % 2 == 1))      # below the diagonal of each pair
        X = X - X @ (torch.where(low, L, 0.0) @ X)
        size *= 2
    return X


def _plain_delta(s):
    c = s["case"]
    T, H, HK, dt, n = c["T"], c["heads"], c["key_heads"], s["o"].dtype, s["lengths"]
    scale = s["scale"]
    q, k = (_in_blocks(s[name], n, HK).repeat_interleave(H // HK, 1) for name in ("q", "k"))
    v, beta = _in_blocks(s["v"], n, H), _in_blocks(s["beta"], n, H)
    g = torch.zeros_like(beta) if s["g"] is None else _in_blocks(s["g"], n, H)
    G = g.double().cumsum(3)                                                    # differences of long sums
    lower = torch.ones((STEPS, STEPS), dtype=torch.bool, device=q.device).tril()
    D = torch.exp(torch.where(lower, G - G.transpose(3, 4), -math.inf)).float()
    y, e, last = torch.exp(G).float(), torch.exp(G[:, :, :, -1:] - G).float(), torch.exp(G[:, :, :, -1:]).float()
    A = (k @ k.transpose(3, 4).contiguous() * D).tril(-1)
    P = q @ k.transpose(3, 4).contiguous() * D
    X = _inverse(beta * A)
    ky, qy, ke = k * y, q * y, k * e
    S = q.new_zeros((*q.shape[:2], c["Dk"], c["Dv"])) if s["S0"] is None else s["S0"]
    O, U, rest, before = torch.empty_like(v), torch.empty_like(v), torch.empty_like(v), []
    for i in range(_blocks(T)):
        before.append(S)
        rest[:, :, i] = v[:, :, i] - ky[:, :, i] @ S
        U[:, :, i] = X[:, :, i] @ (beta[:, :, i] * rest[:, :, i])
        O[:, :, i] = scale * (qy[:, :, i] @ S + P[:, :, i] @ U[:, :, i])
        S = last[:, :, i] * S + ke[:, :, i].transpose(2, 3) @ U[:, :, i]
    o = _in_steps(O, T).to(dt)
    if not c["train"]:
        return dict(o=o, ST=S)
    do = _in_blocks(s["do"], n, H) * scale
    dS, dR, behind = s["dST"], torch.empty_like(v), []
    for i in range(_blocks(T) - 1, -1, -1):
        behind.insert(0, dS)
        dU = P[:, :, i].transpose(2, 3) @ do[:, :, i] + ke[:, :, i] @ dS
        dR[:, :, i] = X[:, :, i].transpose(2, 3) @ dU
        dS = last[:, :, i] * dS + qy[:, :, i].transpose(2, 3) @ do[:, :, i] - (ky[:, :, i] * beta[:, :, i]).transpose(2, 3) @ dR[:, :, i]
    St, dSt = torch.stack(before, 2).transpose(3, 4).contiguous(), torch.stack(behind, 2)
    Ut = U.transpose(3, 4).contiguous()
    dP = (do @ Ut * D).tril()
    dL = (dR @ Ut * D).tril(-1).neg()
    doS, dRS, UdS = do @ St, dR @ St, U @ dSt.transpose(3, 4).contiguous()
    both = beta * dL
    dq = y * doS + dP @ k
    dk = dP.transpose(3, 4).contiguous() @ q + both @ k + both.transpose(3, 4).contiguous() @ k + e * UdS - y * beta * dRS
    kk, qk = k @ k.transpose(3, 4).contiguous(), q @ k.transpose(3, 4).contiguous()
    dbeta = (dR * rest).sum(4, keepdim=True) + (dL * kk).sum(4, keepdim=True)
    pairs = (both * kk + dP * qk).double()
    to_last = (ke * UdS).double().sum(4, keepdim=True)
    dG = pairs.sum(4, keepdim=True) - pairs.sum(3, keepdim=True).transpose(3, 4) - to_last
    dG += (qy * doS).double().sum(4, keepdim=True) - (ky * beta * dRS).double().sum(4, keepdim=True)
    dG[:, :, :, -1:] += to_last.sum(3, keepdim=True) + last.double() * (dSt * St.transpose(3, 4)).double().sum((3, 4), keepdim=True)
    dg = dG.flip(3).cumsum(3).flip(3).float()
    B = c["B"]
    dq, dk = (x.view(B, HK, H // HK, *x.shape[2:]).sum(2) for x in (dq, dk))
    dv = beta * dR
    if n is not None:
        inside = (torch.arange(_blocks(T) * STEPS, device=n.device) < n[:, None]).view(B, 1, -1, STEPS, 1)
        dg, dbeta = torch.where(inside, dg, 0.0), torch.where(inside, dbeta, 0.0)
    return _delta_outputs(o, S, _in_steps(dq, T).to(dt), _in_steps(dk, T).to(dt), _in_steps(dv, T).to(dt),
                          _in_steps(dg, T) if c["decay"] else None, _in_steps(dbeta, T), dS)


def _plain_score(s):
    V, n = s["case"]["V"], s["case"]["top"]
    value = s["logits"].float()
    there = ~torch.isnan(value) & (value > -math.inf)
    if s["allowed"] is not None:
        there &= s["allowed"] != 0
    value = torch.where(there, value, -math.inf)
    biggest = value.amax(1, keepdim=True)
    some = biggest > -math.inf
    d = torch.where(there, value - biggest, 0.0)
    w = torch.where(there, torch.exp(d), 0.0)
    total = w.sum(1, keepdim=True, dtype=torch.float64)
    mean = (w * d).sum(1, keepdim=True, dtype=torch.float64) / torch.where(some, total, 1.0)
    log_total = torch.log(torch.where(some, total, 1.0))
    entropy = (log_total - mean)[:, 0].float()
    given = (s["token"] >= 0) & (s["token"] < V)
    at = torch.where(given, s["token"], 0).long()[:, None]
    mine = value.gather(1, at)
    logprob = torch.where(given, (mine - biggest - log_total)[:, 0].float(), 0.0)
    place = torch.arange(V, device=value.device)[None]
    front = ((value > mine) | ((value == mine) & (place < at))) & there
    rank = torch.where(given, front.sum(1), -1).to(torch.int32)
    top_token = top_logprob = dlogits = None
    if n:
        sorted_value, index = torch.sort(value, dim=1, descending=True, stable=True)
        sorted_value, index = sorted_value[:, :n], index[:, :n]
        top_logprob = (sorted_value - biggest - log_total).float()
        top_token = torch.where(sorted_value > -math.inf, index, -1).to(torch.int32)
    if s["case"]["train"]:
        log_p = (d - log_total).float()
        p = torch.exp(log_p)
        dlp = torch.where(given, s["dlogprob"], 0.0)[:, None]
        dl = -p * (dlp + s["dentropy"][:, None] * (log_p + entropy[:, None]))
        dlogits = torch.where(there, dl.scatter_add_(1, at, dlp), 0.0).to(s["logits"].dtype)
    return _score_outputs(logprob, rank, entropy, top_token, top_logprob, dlogits)


def _plain_distill(s):
    c = s["case"]
    heat = c["temperature"]
    top = s["top_token"].long()
    z = s["top_logit"].double() / heat
    lse_t = s["teacher_lse"].double()[:, None] if c["rest"] else torch.log(torch.exp(z - z.amax(1, keepdim=True)).sum(1, keepdim=True)) + z.amax(1, keepdim=True)
    log_t = z - lse_t
    t = torch.exp(log_t)
    x = s["logits"].float() / heat
    d = x - x.amax(1, keepdim=True)
    w = torch.exp(d)
    log_total = torch.log(w.sum(1, keepdim=True, dtype=torch.float64))
    loss = (t * (log_t - (d.gather(1, top) - log_total))).sum(1)
    share = 0.0
    if c["rest"]:
        t_rest = (1 - t.sum(1, keepdim=True)).clamp_min(0)
        log_rest = torch.log(w.scatter(1, top, 0.0).sum(1, keepdim=True, dtype=torch.float64))
        tail = torch.where(t_rest > 0, t_rest * (torch.log(t_rest) - (log_rest - log_total)), 0.0)
        loss = loss + tail[:, 0]
        share = torch.where(t_rest > 0, t_rest * torch.exp(-(log_rest - log_total)), 0.0).float()       # what is left of 1 - t_rest / s_rest
    loss = (loss * heat ** 2).float()
    if not c["train"]:
        return loss
    p = torch.exp((d - log_total).float())
    dl = p * (1 - share)
    dl.scatter_(1, top, p.gather(1, top) - t.float())
    return loss, (dl * (heat * s["dloss"][:, None])).to(s["logits"].dtype)


_PLAIN = {"delta": _plain_delta, "score": _plain_score, "distill": _plain_distill}
_OWN = {"delta": _own_delta, "score": _own_score, "distill": _own_distill}


# ---- what a pass cannot do without ---------------------------------------------------------------------------------------

def work(case):
    c = case
    size = 2 if c["dtype"] == "bf16" else 4
    if c["kind"] == "delta":
        steps = c["T"] * c["B"]
        keys, values, gates = steps * c["key_heads"] * c["Dk"], steps * c["heads"] * c["Dv"], steps * c["heads"] * (1 + c["decay"])
        states = c["B"] * c["heads"] * c["Dk"] * c["Dv"]
        b, f = 2.0 * size * (keys + values) + 4 * gates + 4.0 * states * (1 + c["state"]), 7.0 * steps * c["heads"] * c["Dk"] * c["Dv"]
        if c["train"]:      # gradients of queries, keys, values, gates and the first state; those of the output and of the last state
            b, f = b + 2.0 * size * (keys + values) + 4 * gates + 8.0 * states, 3 * f
        return {"bytes": b, "flops": f}
    n = float(c["M"]) * c["V"]
    if c["kind"] == "score":
        b = n * (size * (1 + c["train"]) + c["masked"]) + c["M"] * (16.0 + 8 * c["top"])
        return {"bytes": b, "flops": n * (16.0 if c["train"] else 8.0)}
    return {"bytes": n * size * (1.0 + c["train"]) + c["M"] * (8.0 + 8 * c["K"]), "flops": n * (12.0 if c["train"] else 6.0)}


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------------

def exact(case, seed):
    c = case
    if c["kind"] == "delta" and float(c["T"]) * c["B"] * c["heads"] * c["Dk"] * c["Dv"] > 4e10:
        return None
    s = prepare(case, seed)
    return {"delta": _exact_delta, "score": _exact_score, "distill": _exact_distill}[case["kind"]](s, case)


def _exact_delta(s, c):
    """Step after step: S decays, the value that the key finds moves towards the new one, the query reads."""
    T, B, H, HK, Dk, Dv, scale = c["T"], c["B"], c["heads"], c["key_heads"], c["Dk"], c["Dv"], s["scale"]
    dev, group = s["q"].device, H // HK
    on = torch.ones((T, B, 1), dtype=torch.bool, device=dev)
    if s["lengths"] is not None:
        on = (torch.arange(T, device=dev)[:, None] < s["lengths"][None])[:, :, None]

    def key(x, t):
        return torch.where(on[t][:, :, None], x[t].double().reshape(B, HK, Dk), 0.0).repeat_interleave(group, 1)

    def value(x, t):
        return torch.where(on[t][:, :, None], x[t].double().reshape(B, H, Dv), 0.0)

    def gates(t):
        b = torch.where(on[t], s["beta"][t].double(), 0.0)[:, :, None]
        g = torch.zeros_like(b) if s["g"] is None else torch.where(on[t], s["g"][t].double(), 0.0)[:, :, None]
        return b, torch.exp(g)

    def found(S, x):        # x^T S
        return (x[:, :, None] @ S)[:, :, 0]

    def step(S, t):
        k, (b, a) = key(s["k"], t), gates(t)
        S = a[..., None] * S
        u = b * (value(s["v"], t) - found(S, k))
        return S + k[..., None] * u[:, :, None]

    S = torch.zeros((B, H, Dk, Dv), dtype=torch.float64, device=dev) if s["S0"] is None else s["S0"].double()
    o = torch.zeros((T, B, H * Dv), dtype=torch.float64, device=dev)
    marks = []
    for t in range(T):
        if t % 32 == 0:
            marks.append(S.clone() if c["train"] else None)
        S = step(S, t)
        o[t] = (scale * found(S, key(s["q"], t))).reshape(B, H * Dv)
    if not c["train"]:
        return dict(o=o, ST=S)
    dq, dk = (torch.zeros((T, B, HK * Dk), dtype=torch.float64, device=dev) for _ in range(2))
    dv = torch.zeros((T, B, H * Dv), dtype=torch.float64, device=dev)
    dg, dbeta = (torch.zeros((T, B, H), dtype=torch.float64, device=dev) for _ in range(2))
    dS = s["dST"].double()
    for m in range(len(marks) - 1, -1, -1):
        inside = [marks[m]]
        for t in range(32 * m, min(T, 32 * m + 32)):
            inside.append(step(inside[-1], t))
        for t in range(min(T, 32 * m + 32) - 1, 32 * m - 1, -1):
            S1, S0 = inside.pop(), inside[-1]
            k, q, (b, a), d = key(s["k"], t), key(s["q"], t), gates(t), value(s["do"], t)
            dS = dS + scale * q[..., None] * d[:, :, None]
            dq_t = scale * (S1 @ d[..., None])[..., 0]
            Sa = a[..., None] * S0
            miss = value(s["v"], t) - found(Sa, k)
            du = found(dS, k)
            dk_t = (dS @ (b * miss)[..., None])[..., 0] - b * (Sa @ du[..., None])[..., 0]
            dbeta[t] = torch.where(on[t], (du * miss).sum(2), 0.0)
            dv[t] = (b * du).reshape(B, H * Dv)
            dSa = dS - (b * k)[..., None] * du[:, :, None]
            dg[t] = torch.where(on[t], (dSa * Sa).sum((2, 3)), 0.0)
            dS = a[..., None] * dSa
            for out, x in ((dq, dq_t), (dk, dk_t)):
                x = torch.where(on[t][:, :, None], x, 0.0)
                out[t] = x.reshape(B, HK, group, Dk).sum(2).reshape(B, HK * Dk)
        marks[m] = None
    return _delta_outputs(o, S, dq, dk, dv, dg if c["decay"] else None, dbeta, dS)


def _parts(M, V):
    """Runs of rows that fit 64-bit intermediates."""
    n = max(1, (1 << 26) // V)
    return [slice(i, min(M, i + n)) for i in range(0, M, n)]


def _exact_score(s, c):
    M, n = c["M"], c["top"]
    got = []
    for rows in _parts(M, c["V"]):
        l = s["logits"][rows].double()
        gone = torch.isnan(l)
        if s["allowed"] is not None:
            gone = gone | (s["allowed"][rows] == 0)
        l = l.masked_fill(gone, -math.inf)
        log_p = l - torch.logsumexp(l, 1, keepdim=True)
        p = torch.exp(log_p)
        plog = torch.where(p > 0, log_p, 0.0)
        entropy = -(p * plog).sum(1)
        token = s["token"][rows].long()
        given = token >= 0
        logprob = torch.where(given, log_p.gather(1, token.clamp_min(0)[:, None])[:, 0], 0.0)
        top = torch.topk(log_p, min(n, c["V"]), 1).values if n else None
        dl = None
        if c["train"]:
            dlp = torch.where(given, s["dlogprob"][rows].double(), 0.0)[:, None]
            hit = torch.zeros_like(l).scatter_(1, token.clamp_min(0)[:, None], 1.0)
            dl = dlp * (hit - p) - s["dentropy"][rows].double()[:, None] * p * (plog + entropy[:, None])
            dl = dl.masked_fill(gone, 0.0)
        got.append((logprob, entropy, top, dl))
    logprob, entropy, top, dl = (torch.cat(x) if x[0] is not None else None for x in zip(*got))
    return _score_outputs(logprob, None, entropy, None, top, dl)


def _exact_distill(s, c):
    heat, losses, grads = c["temperature"], [], []
    for rows in _parts(c["M"], c["V"]):
        top = s["top_token"][rows].long()
        z = s["top_logit"][rows].double() / heat
        if c["rest"]:
            t = torch.exp(z - s["teacher_lse"][rows].double()[:, None])
        else:
            t = torch.softmax(z, 1)
        x = s["logits"][rows].double() / heat
        log_s = x - torch.logsumexp(x, 1, keepdim=True)
        listed_ = torch.zeros_like(x, dtype=torch.bool).scatter_(1, top, True)
        target = torch.zeros_like(x).scatter_(1, top, t)
        loss = (target * (torch.where(listed_, target, 1.0).log() - log_s)).sum(1)
        t_rest = (1 - t.sum(1)).clamp_min(0) if c["rest"] else torch.zeros_like(loss)
        log_s_rest = torch.logsumexp(log_s.masked_fill(listed_, -math.inf), 1)
        some = t_rest > 0
        loss = loss + torch.where(some, t_rest * (torch.where(some, t_rest, 1.0).log() - log_s_rest), 0.0)
        losses.append(loss * heat ** 2)
        if c["train"]:
            inner = torch.exp(log_s.masked_fill(listed_, -math.inf) - log_s_rest[:, None])      # shares of the words outside the list
            wanted = torch.where(listed_, target, torch.where(some[:, None], t_rest[:, None] * inner, 0.0))
            grad = torch.exp(log_s) - wanted
            if not c["rest"]:
                grad = torch.exp(log_s) - target
            grads.append(grad * heat * s["dloss"][rows].double()[:, None])
    return (torch.cat(losses), torch.cat(grads)) if c["train"] else torch.cat(losses)
