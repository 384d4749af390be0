"""The operators of a recurrent language model around the cells: the gated linear recurrence (the cell whose gates read the
input only) with its gradient, the norm between layers, the 8-bit product and the draw of the next token, as cases that can
be timed.  `own` says whether run() makes the library's calls or computes the plain forms: elementary tensor operations in
32 bits (64 where a border decides), rounded once at the end.

listed() names the cases, draw() gives more of the same ranges, prepare() builds what a user's program holds before the call,
run() is one pass, exact() the same outputs from the definitions in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

BLOCK = 128            # columns that share one scale of an 8-bit operand
E4M3_MAX = 448.0
SMALLEST_SCALE = 2.0 ** -126
STATE_STEPS = 16       # the recurrence's forward keeps one state for so many steps where a gradient is wanted
EPS = 1e-5

# Widths of the latency profile, speech and language-model batches, utterances and word sequences up to documents
UNITS = (64, 2048)
BATCH = (1, 64)
STEPS = (1, 8192)
MAX_CELLS = 1024 * 32 * 2048
ROWS = (1, 16384)
NORM_WIDTH = (64, 8192)
MAX_NORM = 16384 * 2048
PRODUCT_N = (64, 16384)
PRODUCT_K = (64, 8192)
MAX_PRODUCT = 16384 * 8192 * 2048
SEQUENCES = (1, 512)
VOCABULARY = (256, 131072)
MAX_LOGITS = 256 * 32000


def _scan(name, T, B, H, dtype, train=False, reverse=False, ragged=False, state=True):
    return _named(name, kind="scan", T=T, B=B, H=H, dtype=dtype, train=train, reverse=reverse, ragged=ragged, state=state)


def _norm(name, M, N, dtype, residual=True, eight=True, backward=False):
    return _named(name, kind="norm", M=M, N=N, dtype=dtype, residual=residual, eight=eight, backward=backward)


def _product(name, M, N, K, out, quantize=False, w_rows=128, bias=False):
    return _named(name, kind="product", M=M, N=N, K=K, out=out, quantize=quantize, w_rows=w_rows, bias=bias)


def _sample(name, M, V, dtype, top_k=0, top_p=1.0, min_p=0.0, temperature=1.0, mixed=False, masked=False):
    return _named(name, kind="sample", M=M, V=V, dtype=dtype, top_k=top_k, top_p=top_p, min_p=min_p, temperature=temperature,
                  mixed=mixed, masked=masked)


def _named(name, **c):
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token of one user through the recurrence of the 1500-unit language model: latency alone
        _scan("scan_step_b1_h1500", 1, 1, 1500, "f32"),
        # a document read in one go by the same layer, one sequence: few units, many steps
        _scan("scan_long_b1_t8192", 8192, 1, 1500, "bf16"),
        # the backward direction of a bidirectional speech layer over a batch of utterances of different length
        _scan("scan_speech_b16_t300", 300, 16, 800, "f32", reverse=True, ragged=True, state=False),
        # a training step's recurrence: forward and gradient
        _scan("scan_train_b32_t1024", 1024, 32, 2048, "bf16", train=True),
        # one token between two layers: residual, norm and 8-bit activations
        _norm("norm_step_1x1500", 1, 1500, "bf16"),
        # the same over the tokens of a prefill
        _norm("norm_prefill_16384x2048", 16384, 2048, "bf16"),
        # the norm's gradient over a speech batch (300 steps of 16), both directions' units
        _norm("norm_backward_4800x1600", 4800, 1600, "f32", eight=False, backward=True),
        # logits of one token over the 10 000 words of the language model
        _product("product_decode_1x10000x1500", 1, 10000, 1500, "f32"),
        # gate pre-activations of 20 sequences of 35 words, activations quantized on the way in
        _product("linear_700x6000x1500", 700, 6000, 1500, "bf16", quantize=True, bias=True),
        # gate pre-activations of a prefill, 2048 units
        _product("product_prefill_16384x8192x2048", 16384, 8192, 2048, "bf16"),
        # next word of one user
        _sample("sample_1x10000", 1, 10000, "f32", top_k=50, top_p=0.95, temperature=0.8),
        # next token of a full batch, each request with settings and a mask of its own
        _sample("sample_256x32000_mixed", 256, 32000, "bf16", mixed=True, masked=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["scan", "scan", "norm", "product", "product", "sample"])
    dtype = rng.choice(["f32", "bf16"])
    if kind == "scan":
        H, B = _log_int(rng, *UNITS), _log_int(rng, *BATCH)
        T = min(_log_int(rng, *STEPS), MAX_CELLS // (2 if dtype == "f32" else 1) // (H * B))
        return _scan(None, T, B, H, dtype, train=rng.random() < 0.4, reverse=rng.random() < 0.3, ragged=rng.random() < 0.3,
                     state=rng.random() < 0.7)
    if kind == "norm":
        N = _log_int(rng, *NORM_WIDTH)
        M = min(_log_int(rng, *ROWS), MAX_NORM // (2 if dtype == "f32" else 1) // N)
        backward = rng.random() < 0.3
        return _norm(None, M, N, dtype, residual=rng.random() < 0.7, eight=not backward and rng.random() < 0.7, backward=backward)
    if kind == "product":
        N, K = _log_int(rng, *PRODUCT_N), _log_int(rng, *PRODUCT_K)
        M = max(1, min(_log_int(rng, *ROWS), MAX_PRODUCT // (N * K)))
        quantize = rng.random() < 0.3
        return _product(None, M, N, K, "bf16" if quantize else dtype, quantize=quantize, w_rows=rng.choice([128, 128, 1]),
                        bias=rng.random() < 0.5)
    V = _log_int(rng, *VOCABULARY)
    return _sample(None, max(1, min(_log_int(rng, *SEQUENCES), MAX_LOGITS // V)), V, dtype,
                   top_k=rng.choice([0, 0, _log_int(rng, 1, 1000)]), top_p=rng.choice([1.0, round(rng.uniform(0.1, 0.99), 3)]),
                   min_p=rng.choice([0.0, 0.0, round(rng.uniform(0.005, 0.2), 3)]), temperature=round(rng.uniform(0.3, 1.5), 2),
                   mixed=rng.random() < 0.5, masked=rng.random() < 0.3)


# ---- inputs --------------------------------------------------------------------------------------------------------------

def _type(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _blocks(n, of=BLOCK):
    return -(-n // of)


def _padded(n, to=16):
    return -(-n // to) * to


def prepare(case, seed):
    dev = torch.device("cuda:0")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    return {"scan": _prepare_scan, "norm": _prepare_norm, "product": _prepare_product, "sample": _prepare_sample}[case["kind"]](
        case, gen, dev)


def _prepare_scan(c, gen, dev):
    T, B, H, dt = c["T"], c["B"], c["H"], _type(c["dtype"])

    def normal(*shape):
        return torch.randn(shape, generator=gen, device=dev)

    # A layer of one direction, or the second of two whose pre-activations and outputs lie side by side
    sides = 2 if c["reverse"] else 1
    wide = torch.zeros((T, B, sides * 4 * H), dtype=dt, device=dev)
    P = wide[:, :, (sides - 1) * 4 * H:]
    P.copy_(normal(T, B, 4 * H))
    # forget gates that remember from a step or two to about a hundred
    P[:, :, :H] += (torch.rand((H,), generator=gen, device=dev) * 4).to(dt)
    s = dict(case=c, P=P, h=torch.empty((T, B, sides * H), dtype=dt, device=dev)[:, :, (sides - 1) * H:], lengths=None,
             c0=normal(B, H) * 0.5 if c["state"] else None, cT=torch.empty((B, H), device=dev))
    if c["ragged"]:
        n = torch.randint(0, T + 1, (B,), generator=gen, device=dev, dtype=torch.int32)
        n[0] = T
        s["lengths"] = n
    if c["train"]:
        s.update(dh=normal(T, B, H).to(dt), dcT=normal(B, H), dP=torch.empty((T, B, 4 * H), dtype=dt, device=dev),
                 dc0=torch.empty((B, H), device=dev),
                 states=torch.empty((_blocks(T, STATE_STEPS), B, H), device=dev))
    return s


def _prepare_norm(c, gen, dev):
    M, N, dt = c["M"], c["N"], _type(c["dtype"])

    def rows(size):
        return (torch.randn((M, N), generator=gen, device=dev) * size).to(dt)

    # a residual stream: some of its columns are far larger than the rest
    columns = torch.exp(0.7 * torch.randn((N,), generator=gen, device=dev))
    s = dict(case=c, weight=1 + 0.2 * torch.randn((N,), generator=gen, device=dev))
    if c["backward"]:
        s["sum"] = rows(columns)
        s["rstd"] = torch.rsqrt(s["sum"].float().square().mean(1) + EPS)
        s.update(dy=rows(0.1), dsum=rows(0.1) if c["residual"] else None, dx=torch.empty((M, N), dtype=dt, device=dev),
                 dweight=torch.empty((N,), device=dev))
        return s
    s.update(x=rows(0.5), residual=rows(columns) if c["residual"] else None, rstd=torch.empty((M,), device=dev),
             sum=torch.empty((M, N), dtype=dt, device=dev) if c["residual"] else None, y=None, y8=None, scale=None)
    if c["eight"]:
        s.update(y8=torch.empty((M, _padded(N)), dtype=torch.float8_e4m3fn, device=dev),
                 scale=torch.empty((M, _blocks(N)), device=dev))
    else:
        s["y"] = torch.empty((M, N), dtype=dt, device=dev)
    return s


def _prepare_product(c, gen, dev):
    M, N, K = c["M"], c["N"], c["K"]

    def eight(v, block_rows):
        q, scale = _quantize(v, block_rows)
        held = torch.zeros((v.shape[0], _padded(K)), dtype=torch.float8_e4m3fn, device=dev)
        held[:, :K] = q
        return held, scale

    x = torch.randn((M, K), generator=gen, device=dev) * torch.exp(0.7 * torch.randn((K,), generator=gen, device=dev))
    W, w_scale = eight(torch.randn((N, K), generator=gen, device=dev) / math.sqrt(K), c["w_rows"])
    s = dict(case=c, W=W, w_scale=w_scale, C=torch.empty((M, N), dtype=_type(c["out"]), device=dev),
             bias=torch.randn((N,), generator=gen, device=dev) * 0.1 if c["bias"] else None)
    if c["quantize"]:
        s.update(x=x.bfloat16(), A=torch.zeros((M, _padded(K)), dtype=torch.float8_e4m3fn, device=dev),
                 a_scale=torch.empty((M, _blocks(K)), device=dev))
    else:
        s["A"], s["a_scale"] = eight(x, 1)
    return s


def _prepare_sample(c, gen, dev):
    M, V = c["M"], c["V"]

    def uniform(*shape):
        return torch.rand(shape, generator=gen, device=dev)

    s = dict(case=c, logits=(torch.randn((M, V), generator=gen, device=dev) * 2.5).to(_type(c["dtype"])), u=uniform(M), allowed=None,
             token=torch.empty((M,), dtype=torch.int32, device=dev), prob=torch.empty((M,), device=dev),
             kept=torch.empty((M,), dtype=torch.int32, device=dev))
    if c["masked"]:     # a grammar or a list of banned words; what is masked holds anything
        s["allowed"] = (uniform(M, V) < 0.8).to(torch.uint8)
        s["logits"][s["allowed"] == 0] = float("nan")
    temperature, top_k, top_p, min_p = (torch.full((M,), c[n], device=dev) for n in ("temperature", "top_k", "top_p", "min_p"))
    if c["mixed"]:      # every request brings its own settings; some want the likeliest token, some no filter at all
        temperature = torch.where(uniform(M) < 0.2, torch.zeros((), device=dev), 0.3 + 1.2 * uniform(M))
        top_k = torch.where(uniform(M) < 0.5, 0.0, torch.exp(uniform(M) * math.log(min(V, 1000))).floor())
        top_p = torch.where(uniform(M) < 0.4, 1.0, 0.5 + 0.49 * uniform(M))
        min_p = torch.where(uniform(M) < 0.6, 0.0, 0.1 * uniform(M))
    s.update(temperature=temperature, top_k=top_k.to(torch.int32), top_p=top_p, min_p=min_p)
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


def _own_scan(s):
    from paper_1901_10997_amd import binding as L
    c, P, h, ptr = s["case"], s["P"], s["h"], _ptr
    T, B, H = c["T"], c["B"], c["H"]
    dtype = L.LSTM_BF16 if c["dtype"] == "bf16" else L.LSTM_F32
    if "ws" not in s:
        _workspace(s, L.lstm_scan_workspace_bytes(T, B, H))
    ws, stream = s["ws"], torch.cuda.current_stream().cuda_stream
    L.lstm_scan_forward(T, B, H, dtype, c["reverse"], ptr(P), P.stride(0), P.stride(1), ptr(s["lengths"]), ptr(s["c0"]), ptr(h),
                        h.stride(0), h.stride(1), ptr(s["cT"]), ptr(s.get("states")), ptr(ws), ws.numel(), stream)
    if not c["train"]:
        return h, s["cT"]
    dh, dP = s["dh"], s["dP"]
    L.lstm_scan_backward(T, B, H, dtype, c["reverse"], ptr(P), P.stride(0), P.stride(1), ptr(s["lengths"]), ptr(s["states"]), ptr(dh),
                         dh.stride(0), dh.stride(1), ptr(s["dcT"]), ptr(dP), dP.stride(0), dP.stride(1), ptr(s["dc0"]), ptr(ws),
                         ws.numel(), stream)
    return h, s["cT"], dP, s["dc0"]


def _own_norm(s):
    from paper_1901_10997_amd import binding as L
    c, ptr = s["case"], _ptr
    M, N = c["M"], c["N"]
    dtype = L.LSTM_BF16 if c["dtype"] == "bf16" else L.LSTM_F32
    stream = torch.cuda.current_stream().cuda_stream
    if c["backward"]:
        if "ws" not in s:
            _workspace(s, L.lstm_rmsnorm_workspace_bytes(M, N))
        L.lstm_rmsnorm_backward(M, N, dtype, ptr(s["sum"]), N, ptr(s["weight"]), ptr(s["rstd"]), ptr(s["dy"]), N, ptr(s["dsum"]), N,
                                ptr(s["dx"]), N, ptr(s["dweight"]), ptr(s["ws"]), s["ws"].numel(), stream)
        return s["dx"], s["dweight"]
    y8 = s["y8"]
    L.lstm_rmsnorm_forward(M, N, dtype, ptr(s["x"]), N, ptr(s["residual"]), N, ptr(s["weight"]), EPS, ptr(s["sum"]), N, ptr(s["y"]), N,
                           ptr(y8), 0 if y8 is None else y8.stride(0), ptr(s["scale"]), _blocks(N), ptr(s["rstd"]), stream)
    return _norm_outputs(s["sum"], s["rstd"], s["y"], None if y8 is None else y8[:, :N], s["scale"])


def _norm_outputs(total, rstd, y, y8, scale):
    out = dict(sum=total, rstd=rstd, y=y, y8=y8, scale=scale)
    return {k: v for k, v in out.items() if v is not None}


def _own_product(s):
    from paper_1901_10997_amd import binding as L
    c, A, W, ptr = s["case"], s["A"], s["W"], _ptr
    M, N, K = c["M"], c["N"], c["K"]
    stream = torch.cuda.current_stream().cuda_stream
    if "ws" not in s:
        _workspace(s, L.lstm_matmul_fp8_workspace_bytes(M, N, K))
    if c["quantize"]:
        L.lstm_quantize_fp8(M, K, L.LSTM_BF16, 1, ptr(s["x"]), K, ptr(A), A.stride(0), ptr(s["a_scale"]), _blocks(K), stream)
    L.lstm_matmul_fp8(M, N, K, ptr(A), A.stride(0), ptr(s["a_scale"]), _blocks(K), ptr(W), W.stride(0), ptr(s["w_scale"]), _blocks(K),
                      c["w_rows"], ptr(s["bias"]), L.LSTM_BF16 if c["out"] == "bf16" else L.LSTM_F32, ptr(s["C"]), N, ptr(s["ws"]),
                      s["ws"].numel(), stream)
    return dict(C=s["C"], A=A[:, :K], scale=s["a_scale"]) if c["quantize"] else s["C"]


def _own_sample(s):
    from paper_1901_10997_amd import binding as L
    c, ptr = s["case"], _ptr
    M, V = c["M"], c["V"]
    if "ws" not in s:
        _workspace(s, L.lstm_sample_workspace_bytes(M, V))
    L.lstm_sample(M, V, L.LSTM_BF16 if c["dtype"] == "bf16" else L.LSTM_F32, ptr(s["logits"]), V, ptr(s["allowed"]), V,
                  ptr(s["temperature"]), ptr(s["top_k"]), ptr(s["top_p"]), ptr(s["min_p"]), ptr(s["u"]), ptr(s["token"]),
                  ptr(s["prob"]), ptr(s["kept"]), ptr(s["ws"]), s["ws"].numel(), torch.cuda.current_stream().cuda_stream)
    return s["token"], s["prob"], s["kept"]


def _flip(v, lengths):
    """Steps t of every sequence in the order in which its own last step comes first (what is behind it stays)."""
    T = v.shape[0]
    if lengths is None:
        return v.flip(0)
    t = torch.arange(T, device=v.device)[:, None]
    at = torch.where(t < lengths, lengths - 1 - t, t)
    return torch.gather(v, 0, at[:, :, None].expand_as(v))


def _linear_scan(a, b):
    """s_t = a_t s_{t-1} + b_t over dimension 0 from zero: after each doubling a and b stand for twice as many steps."""
    step = 1
    while step < a.shape[0]:
        b = torch.cat((b[:step], torch.addcmul(b[step:], a[step:], b[:-step])))
        a = torch.cat((a[:step], a[step:] * a[:-step]))
        step *= 2
    return b


def _plain_scan(s):
    c, dt = s["case"], s["h"].dtype
    T, B, H, n = c["T"], c["B"], c["H"], s["lengths"]
    P = s["P"].float()
    if c["reverse"]:
        P = _flip(P, n)
    f, i, o = (torch.sigmoid(P[:, :, q * H:(q + 1) * H]) for q in range(3))
    g = torch.tanh(P[:, :, 3 * H:])
    inside = None if n is None else (torch.arange(T, device=P.device)[:, None] < n)[:, :, None]
    add = i * g
    if inside is not None:      # a sequence that has ended keeps its state
        f, add = torch.where(inside, f, 1.0), torch.where(inside, add, 0.0)
    c0 = torch.zeros((B, H), device=P.device) if s["c0"] is None else s["c0"]
    cell = _linear_scan(f, torch.cat((torch.addcmul(add[:1], f[:1], c0[None]), add[1:])))
    squashed = torch.tanh(cell)
    h = o * squashed if inside is None else torch.where(inside, o * squashed, 0.0)
    h_out = (_flip(h, n) if c["reverse"] else h).to(dt)
    if not c["train"]:
        return h_out, cell[-1]
    dh = s["dh"].float()
    if c["reverse"]:
        dh = _flip(dh, n)
    if inside is not None:
        dh = torch.where(inside, dh, 0.0)
    into = dh * o * (1 - squashed * squashed)
    into[-1] += s["dcT"]
    next_f = torch.cat((f[1:], torch.zeros_like(f[:1])))
    delta = _linear_scan(next_f.flip(0), into.flip(0)).flip(0)
    before = torch.cat((c0[None], cell[:-1]))
    dP = torch.cat((delta * before * f * (1 - f), delta * g * i * (1 - i), dh * squashed * o * (1 - o), delta * i * (1 - g * g)), 2)
    if inside is not None:
        dP = torch.where(inside, dP, 0.0)
    if c["reverse"]:
        dP = _flip(dP, n)
    return h_out, cell[-1], dP.to(dt), f[0] * delta[0]


def _quantize(v, block_rows):
    """e4m3 values and scales [rows / block_rows, blocks]: the largest magnitude of a block becomes 448."""
    R, K = v.shape
    RB, KB = _blocks(R, block_rows), _blocks(K)
    w = torch.nn.functional.pad(v.float(), (0, KB * BLOCK - K, 0, RB * block_rows - R))
    w = w.view(RB, block_rows, KB, BLOCK)
    scale = (w.abs().amax((1, 3)) / E4M3_MAX).clamp_min(SMALLEST_SCALE)
    q = (w / scale[:, None, :, None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
    return q.view(RB * block_rows, KB * BLOCK)[:R, :K], scale


def _spread(scale, block_rows, R, K):
    """A block's scale in every place of it."""
    return scale.repeat_interleave(BLOCK, 1)[:, :K].repeat_interleave(block_rows, 0)[:R]


def _plain_norm(s):
    c = s["case"]
    dt = _type(c["dtype"])
    if c["backward"]:
        x_hat = s["sum"].float() * s["rstd"][:, None]
        dy = s["dy"].float()
        g = dy * s["weight"]
        dx = s["rstd"][:, None] * (g - x_hat * (g * x_hat).mean(1, keepdim=True))
        if s["dsum"] is not None:
            dx = dx + s["dsum"].float()
        return dx.to(dt), (dy * x_hat).sum(0)
    total = s["x"] if s["residual"] is None else (s["x"].float() + s["residual"].float()).to(dt)
    v = total.float()
    rstd = torch.rsqrt(v.square().mean(1) + EPS)
    y = v * rstd[:, None] * s["weight"]
    y8, scale = _quantize(y, 1) if c["eight"] else (None, None)
    return _norm_outputs(None if s["residual"] is None else total, rstd, None if c["eight"] else y.to(dt), y8, scale)


def _plain_product(s):
    c = s["case"]
    M, N, K = c["M"], c["N"], c["K"]
    A, a_scale = _quantize(s["x"], 1) if c["quantize"] else (s["A"][:, :K], s["a_scale"])
    left = A.float() * _spread(a_scale, 1, M, K)
    right = s["W"][:, :K].float() * _spread(s["w_scale"], c["w_rows"], N, K)
    C = left @ right.t()
    if s["bias"] is not None:
        C = C + s["bias"]
    C = C.to(s["C"].dtype)
    return dict(C=C, A=A, scale=a_scale) if c["quantize"] else C


def _plain_sample(s):
    """In 64 bits: a token is kept or not, and drawn or not, by which side of a border a sum lies."""
    V = s["case"]["V"]
    logits = s["logits"].double()
    if s["allowed"] is not None:
        logits = torch.where(s["allowed"] != 0, logits, -math.inf)
    value, index = torch.sort(logits, dim=1, descending=True, stable=True)
    there = value > -math.inf
    greedy = (s["temperature"] <= 0)[:, None]
    heat = torch.where(greedy, 1.0, s["temperature"].double()[:, None])
    w = torch.where(there, torch.exp((value - value[:, :1]) / heat), 0.0)
    rank = torch.arange(V, device=w.device)[None]
    k = torch.where(s["top_k"] > 0, s["top_k"], V)[:, None]
    keep = there & (rank < torch.where(greedy, 1, k))
    w = torch.where(keep, w, 0.0)
    p = s["top_p"].double()[:, None]
    running = w.cumsum(1)
    keep &= (p >= 1) | (running - w < p * running[:, -1:]) | (rank == 0)
    keep &= w >= s["min_p"].double()[:, None]
    chosen = torch.zeros_like(w).scatter_(1, index, torch.where(keep, w, 0.0))     # back in the order of the vocabulary
    running = chosen.cumsum(1)
    total = running[:, -1:]
    past = running > s["u"].double()[:, None] * total
    token = past.to(torch.uint8).argmax(1)
    some = total[:, 0] > 0
    prob = chosen.gather(1, token[:, None])[:, 0] / torch.where(some, total[:, 0], 1.0)
    return torch.where(some, token, -1).to(torch.int32), prob.float(), keep.sum(1).to(torch.int32)


_PLAIN = {"scan": _plain_scan, "norm": _plain_norm, "product": _plain_product, "sample": _plain_sample}
_OWN = {"scan": _own_scan, "norm": _own_norm, "product": _own_product, "sample": _own_sample}


# ---- what a pass cannot do without ---------------------------------------------------------------------------------------

def work(case):
    c = case
    size = 2 if c.get("dtype") == "bf16" else 4
    if c["kind"] == "scan":
        cells, states = c["T"] * c["B"] * c["H"], c["B"] * c["H"]
        b, f = 5.0 * size * cells + 4 * states * (1 + c["state"]), 30.0 * cells
        if c["train"]:      # and again the pre-activations, the gradient of h and that of the pre-activations; one state in 16
            b, f = b + 9.0 * size * cells + 8.0 * states * _blocks(c["T"], STATE_STEPS) + 8.0 * states, f + 60.0 * cells
        return {"bytes": b, "flops": f}
    if c["kind"] == "norm":
        n = c["M"] * c["N"]
        if c["backward"]:
            return {"bytes": n * size * (3.0 + c["residual"]) + 8.0 * c["N"] + 4.0 * c["M"], "flops": 12.0 * n}
        return {"bytes": n * (size * (1.0 + 2 * c["residual"]) + (1 if c["eight"] else size)) + 4.0 * c["N"] + 4.0 * c["M"], "flops": 8.0 * n}
    if c["kind"] == "product":
        M, N, K = c["M"], c["N"], c["K"]
        out = 2 if c["out"] == "bf16" else 4
        scales = 4.0 * _blocks(K) * (M + _blocks(N, c["w_rows"]))
        return {"bytes": float(N) * K + M * K * (3.0 if c["quantize"] else 1.0) + M * N * float(out) + scales, "flops": 2.0 * M * N * K}
    return {"bytes": float(c["M"]) * c["V"] * (size + c["masked"]), "flops": 8.0 * c["M"] * c["V"]}


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"scan": _exact_scan, "norm": _exact_norm, "product": _exact_product, "sample": _exact_sample}[case["kind"]](s, case)


def _exact_scan(s, c):
    """Step after step, each sequence in its own order."""
    T, B, H = c["T"], c["B"], c["H"]
    dev = s["P"].device
    P = s["P"].double()
    f, i, o = (1 / (1 + torch.exp(-P[:, :, q * H:(q + 1) * H])) for q in range(3))
    g = torch.tanh(P[:, :, 3 * H:])
    del P
    length = torch.full((B,), T, device=dev) if s["lengths"] is None else s["lengths"].long()
    row = torch.arange(B, device=dev)
    state = torch.zeros((B, H), dtype=torch.float64, device=dev) if s["c0"] is None else s["c0"].double()
    h = torch.zeros((T, B, H), dtype=torch.float64, device=dev)
    cells = torch.empty_like(h) if c["train"] else None      # the state in front of each step
    whole = s["lengths"] is None

    def place(t):
        return (T - 1 - t if c["reverse"] else t) if whole else torch.where(length > t, length - 1 - t if c["reverse"] else t, t)

    def at(v, t):
        p = place(t)
        return v[p] if whole else v[p, row]

    for t in range(T):
        new = at(f, t) * state + at(i, t) * at(g, t)
        out = at(o, t) * torch.tanh(new)
        if cells is not None:
            cells[t] = state
        if whole:
            h[place(t)], state = out, new
        else:
            on = (length > t)[:, None]
            h[place(t), row] = torch.where(on, out, 0.0)
            state = torch.where(on, new, state)
    if not c["train"]:
        return h, state
    dP = torch.zeros((T, B, 4 * H), dtype=torch.float64, device=dev)
    carry = s["dcT"].double()
    dh_all = s["dh"]
    for t in range(T - 1, -1, -1):
        p = place(t)
        F, I, O, G, dh = at(f, t), at(i, t), at(o, t), at(g, t), at(dh_all, t).double()
        tc = torch.tanh(F * cells[t] + I * G)
        delta = carry + dh * O * (1 - tc ** 2)
        d = torch.cat((delta * cells[t] * F * (1 - F), delta * G * I * (1 - I), dh * tc * O * (1 - O), delta * I * (1 - G ** 2)), 1)
        if whole:
            dP[p], carry = d, delta * F
        else:
            on = (length > t)[:, None]
            dP[p, row] = torch.where(on, d, 0.0)
            carry = torch.where(on, delta * F, carry)
    return h, state, dP, carry


def _exact_eight(v):
    """What an e4m3 code stands for before it is rounded, and the scale."""
    R, K = v.shape
    scale = torch.stack([part.abs().amax(1) for part in v.split(BLOCK, 1)], 1) / E4M3_MAX
    scale = scale.clamp_min(SMALLEST_SCALE)
    return v / scale[:, torch.arange(K, device=v.device) // BLOCK], scale


def _exact_norm(s, c):
    N = c["N"]
    if c["backward"]:
        x, dy, w = s["sum"].double(), s["dy"].double(), s["weight"].double()
        r = s["rstd"].double()[:, None]
        inner = (dy * w * x).sum(1, keepdim=True)
        dx = r * dy * w - x * r ** 3 * inner / N
        return dx if s["dsum"] is None else dx + s["dsum"].double(), torch.einsum("mn,mn->n", dy, x * r)
    total = s["x"].double() if s["residual"] is None else (s["x"].double() + s["residual"].double()).to(s["x"].dtype).double()
    rstd = 1 / torch.sqrt((total ** 2).sum(1) / N + EPS)
    y = total * rstd[:, None] * s["weight"].double()
    y8, scale = _exact_eight(y) if c["eight"] else (None, None)
    return _norm_outputs(None if s["residual"] is None else total, rstd, None if c["eight"] else y, y8, scale)


def _exact_product(s, c):
    """Block after block of 128 columns, each with its scales."""
    M, N, K = c["M"], c["N"], c["K"]
    if float(M) * N * K > 4e11:
        return None
    dev = s["W"].device
    if c["quantize"]:
        unrounded, scale = _exact_eight(s["x"].double())
        A = unrounded.float().clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn).double()
    else:
        unrounded, scale, A = None, s["a_scale"].double(), s["A"].double()
    W, w_scale = s["W"].double(), s["w_scale"].double()
    w_row = torch.arange(N, device=dev) // c["w_rows"]
    C = torch.zeros((M, N), dtype=torch.float64, device=dev)
    for b in range(_blocks(K)):
        cols = slice(b * BLOCK, min(K, (b + 1) * BLOCK))
        C += scale[:, b, None] * w_scale[w_row, b] * (A[:, cols] @ W[:, cols].t())
    if s["bias"] is not None:
        C += s["bias"].double()
    return dict(C=C, A=unrounded, scale=scale) if c["quantize"] else C


def _exact_sample(s, c):
    """Row by row: who comes before whom, who is kept, and a walk down the vocabulary; the probability of what it draws."""
    prob = torch.zeros((c["M"],), dtype=torch.float64, device=s["logits"].device)
    for m in range(c["M"]):
        l = s["logits"][m].double()
        if s["allowed"] is not None:
            l = l.masked_fill(s["allowed"][m] == 0, -math.inf)
        top = l.max()
        if not bool(top > -math.inf):
            continue
        if float(s["temperature"][m]) <= 0:
            prob[m] = 1.0
            continue
        w = torch.exp((l - top) / s["temperature"][m].double())
        order = torch.argsort(-l, stable=True)
        k = int(s["top_k"][m])
        order = order[: k if k > 0 else c["V"]]
        mass, p = w[order], float(s["top_p"][m])
        if p < 1:
            before = mass.cumsum(0) - mass
            order = order[: max(1, int((before < p * mass.sum()).sum()))]
        order = order[w[order] >= s["min_p"][m].double()].sort().values
        walked = w[order].cumsum(0)
        drawn = int(torch.searchsorted(walked, (s["u"][m].double() * walked[-1])[None], right=True)[0])
        prob[m] = w[order[drawn]] / walked[-1]
    return None, prob, None
