"""The operators around the cells in numpy and 64 bits, from their formulas: gated linear recurrence and its gradient, RMS
norm and its gradient, e4m3 quantization, the product with block scales, the draw of a token, the gated delta rule and its
gradient, scores of tokens and the distillation loss with their gradients.  Test infrastructure."""
from __future__ import annotations

import math

import numpy as np

BLOCK = 128
E4M3_MAX = 448.0
SMALLEST_SCALE = np.float32(2.0 ** -126)


def sigmoid(z):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-np.asarray(z, np.float64)))


def _places(T, length, reverse):
    return [length - 1 - s if reverse else s for s in range(length)]


def scan_forward(P, lengths=None, c0=None, reverse=False):
    """P [T, B, 4H].  Returns h [T, B, H], cT [B, H], the state in front of every step by step number [T, B, H]."""
    T, B, H4 = P.shape
    H = H4 // 4
    h, before = np.zeros((T, B, H)), np.zeros((T, B, H))
    state = np.zeros((B, H)) if c0 is None else np.array(c0, np.float64)
    for b in range(B):
        n = T if lengths is None else min(max(int(lengths[b]), 0), T)
        for s, t in enumerate(_places(T, n, reverse)):
            p = np.asarray(P[t, b], np.float64).reshape(4, H)
            before[s, b] = state[b]
            state[b] = sigmoid(p[0]) * state[b] + sigmoid(p[1]) * np.tanh(p[3])
            h[t, b] = sigmoid(p[2]) * np.tanh(state[b])
        before[n:, b] = state[b]
    return h, state, before


def scan_backward(P, before, dh, dcT=None, lengths=None, reverse=False):
    """dP [T, B, 4H] and dc0 [B, H] from the states scan_forward returned."""
    T, B, H4 = P.shape
    H = H4 // 4
    dP = np.zeros((T, B, H4))
    carry = np.zeros((B, H)) if dcT is None else np.array(dcT, np.float64)
    for b in range(B):
        n = T if lengths is None else min(max(int(lengths[b]), 0), T)
        places = _places(T, n, reverse)
        for s in range(n - 1, -1, -1):
            t = places[s]
            p = np.asarray(P[t, b], np.float64).reshape(4, H)
            f, i, o, g = sigmoid(p[0]), sigmoid(p[1]), sigmoid(p[2]), np.tanh(p[3])
            tc = np.tanh(f * before[s, b] + i * g)
            d = np.asarray(dh[t, b], np.float64)
            delta = carry[b] + d * o * (1 - tc * tc)
            dP[t, b] = np.concatenate((delta * before[s, b] * f * (1 - f), delta * g * i * (1 - i), d * tc * o * (1 - o),
                                       delta * i * (1 - g * g)))
            carry[b] = f * delta
    return dP, carry


def rmsnorm(s, weight, eps):
    s = np.asarray(s, np.float64)
    rstd = 1.0 / np.sqrt((s * s).mean(1) + eps)
    return s * rstd[:, None] * (1.0 if weight is None else np.asarray(weight, np.float64)), rstd


def rmsnorm_backward(s, weight, rstd, dy, dsum):
    s, dy, rstd = np.asarray(s, np.float64), np.asarray(dy, np.float64), np.asarray(rstd, np.float64)[:, None]
    x = s * rstd
    g = dy if weight is None else dy * np.asarray(weight, np.float64)
    dx = rstd * (g - x * (g * x).mean(1, keepdims=True))
    return (dx if dsum is None else dx + np.asarray(dsum, np.float64)), (dy * x).sum(0)


def _e4m3_values():
    """The 127 non-negative values by code: 3 bits of mantissa, exponent bias 7, code 127 is NaN."""
    return np.array([(8 + (q & 7)) * 2.0 ** ((q >> 3) - 10) if q >> 3 else (q & 7) * 2.0 ** -9 for q in range(127)])


_VALUES = _e4m3_values()
_BETWEEN = (_VALUES[1:] + _VALUES[:-1]) / 2


def e4m3_encode(v):
    """Codes of values of magnitude up to 464, nearest, ties to the even code; NaN is code 127."""
    v = np.asarray(v, np.float64)
    mag = np.abs(v)
    low = np.searchsorted(_BETWEEN, mag, side="left")        # first code whose upper border is not below
    tie = (low < len(_BETWEEN)) & (mag == _BETWEEN[np.minimum(low, len(_BETWEEN) - 1)])
    code = np.where(tie & (low % 2 == 1), low + 1, low)
    code = np.where(np.isnan(v), 127, code)
    return (code | np.where(np.signbit(v), 128, 0)).astype(np.uint8)


def e4m3_decode(code):
    code = np.asarray(code)
    table = np.append(_VALUES, np.nan)
    return np.where(code & 128, -1.0, 1.0) * table[code & 127]


def _blocks(n, of=BLOCK):
    return -(-n // of)


def spread(scale, block_rows, R, K):
    return np.repeat(np.repeat(scale, BLOCK, 1)[:, :K], block_rows, 0)[:R]


def quantize(x, block_rows=1):
    """Codes and fp32 scales with the arithmetic of the definition in fp32: one division for the scale, one for the value."""
    x = np.asarray(x, np.float32)
    R, K = x.shape
    RB, KB = _blocks(R, block_rows), _blocks(K)
    scale = np.empty((RB, KB), np.float32)
    for i in range(RB):
        for j in range(KB):
            mag = np.abs(x[i * block_rows:(i + 1) * block_rows, j * BLOCK:(j + 1) * BLOCK])
            mag = mag[~np.isnan(mag)]
            top = np.float32(min(mag.max(initial=np.float32(0)), np.finfo(np.float32).max))
            scale[i, j] = max(top / np.float32(E4M3_MAX), SMALLEST_SCALE)
    with np.errstate(over="ignore", invalid="ignore"):
        v = x / spread(scale, block_rows, R, K)
        v = np.where(np.abs(v) > E4M3_MAX, np.copysign(np.float32(E4M3_MAX), v), v)
    return e4m3_encode(v), scale


def matmul(A, a_scale, W, w_scale, w_block_rows, bias=None):
    """Product of codes, and the sum of the magnitudes of its terms."""
    (M, K), N = A.shape, W.shape[0]
    a = e4m3_decode(A) * spread(np.asarray(a_scale, np.float64), 1, M, K)
    w = e4m3_decode(W) * spread(np.asarray(w_scale, np.float64), w_block_rows, N, K)
    C = a @ w.T
    size = np.abs(a) @ np.abs(w).T
    return (C, size) if bias is None else (C + np.asarray(bias, np.float64), size + np.abs(np.asarray(bias, np.float64)))


def sample(logits, u, allowed=None, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """One row: token, its probability and how many stayed.  u, temperature, top_p and min_p are the fp32 values."""
    l = np.asarray(logits, np.float64)
    there = ~np.isnan(l) & (l > -np.inf)
    if allowed is not None:
        there &= np.asarray(allowed) != 0
    index = np.nonzero(there)[0]
    if not len(index):
        return -1, 0.0, 0
    order = index[np.argsort(-l[index], kind="stable")]
    if not temperature > 0:
        return int(order[0]), 1.0, 1
    top = l[order[0]]
    with np.errstate(invalid="ignore"):
        w = np.where(l[order] == top, 1.0, np.exp((l[order] - top) / float(temperature)))
    if top_k > 0:
        order, w = order[:top_k], w[:top_k]
    if top_p < 1:
        total, stay, front = math.fsum(w), 0, []
        while stay < len(w) and (stay == 0 or math.fsum(front) < float(top_p) * total):
            front.append(w[stay])
            stay += 1
        order, w = order[:stay], w[:stay]
    stay = w >= min(float(min_p), 1.0)
    order, w = order[stay], w[stay]
    by_index = np.argsort(order)
    order, w = order[by_index], w[by_index]
    want = float(u) * math.fsum(w)
    run = 0.0
    for j, v in zip(order, w):
        run = run + v
        if run > want:
            return int(j), float(v / math.fsum(w)), len(order)
    return int(order[-1]), float(w[-1] / math.fsum(w)), len(order)


# ---- gated delta rule: S_t = a_t (I - b_t k_t k_t') S_{t-1} + b_t k_t v_t', o_t = scale S_t' q_t

def _delta_rows(x, T, B, heads):
    return np.asarray(x, np.float64).reshape(T, B, heads, -1)


def _delta_inside(T, B, lengths):
    n = np.full(B, T) if lengths is None else np.clip(np.asarray(lengths), 0, T)
    return np.arange(T)[:, None] < n[None]


def delta_forward(q, k, v, g, beta, heads, key_heads, scale, lengths=None, S0=None):
    """q, k [T, B, key_heads * Dk], v [T, B, heads * Dv], g (log decay) or None, beta [T, B, heads].  Returns o, the final state and
    the state in front of every step [T, B, heads, Dk, Dv].  What stands behind a sequence's end is not looked at."""
    T, B = beta.shape[:2]
    q, k, v = _delta_rows(q, T, B, key_heads), _delta_rows(k, T, B, key_heads), _delta_rows(v, T, B, heads)
    q, k = (np.repeat(x, heads // key_heads, axis=2) for x in (q, k))
    inside = _delta_inside(T, B, lengths)
    S = np.zeros((B, heads, q.shape[3], v.shape[3])) if S0 is None else np.array(S0, np.float64)
    o, front = np.zeros((T, B, heads, v.shape[3])), np.zeros((T,) + S.shape)
    for t in range(T):
        front[t] = S
        for b in np.flatnonzero(inside[t]):
            a = np.ones(heads) if g is None else np.exp(np.asarray(g[t, b], np.float64))
            S[b] *= a[:, None, None]
            u = np.asarray(beta[t, b], np.float64)[:, None] * (v[t, b] - np.einsum("hd,hdv->hv", k[t, b], S[b]))
            S[b] += np.einsum("hd,hv->hdv", k[t, b], u)
            o[t, b] = scale * np.einsum("hd,hdv->hv", q[t, b], S[b])
    return o.reshape(T, B, -1), S, front


def delta_backward(q, k, v, g, beta, heads, key_heads, scale, front, dO, lengths=None, dST=None, sizes=None):
    """Gradients dq, dk, dv, dg, dbeta, dS0 from the states delta_forward returned; 0 behind a sequence's end.  sizes: a dict that
    receives for dg and dbeta, which are inner products, the product of the lengths or the sum of the magnitudes."""
    T, B = beta.shape[:2]
    q, k, v, dO = _delta_rows(q, T, B, key_heads), _delta_rows(k, T, B, key_heads), _delta_rows(v, T, B, heads), _delta_rows(dO, T, B, heads)
    group = heads // key_heads
    inside = _delta_inside(T, B, lengths)
    dq, dk, dv, dg, db = np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape), np.zeros((T, B, heads)), np.zeros((T, B, heads))
    D = np.zeros(front.shape[1:]) if dST is None else np.array(dST, np.float64)
    if sizes is not None:
        sizes.update(dg=np.zeros(dg.shape), dbeta=np.zeros(db.shape))
    for t in range(T - 1, -1, -1):
        for b in np.flatnonzero(inside[t]):
            K, Q = np.repeat(k[t, b], group, axis=0), np.repeat(q[t, b], group, axis=0)
            a = np.ones(heads) if g is None else np.exp(np.asarray(g[t, b], np.float64))
            bt = np.asarray(beta[t, b], np.float64)
            decayed = a[:, None, None] * front[t, b]
            miss = v[t, b] - np.einsum("hd,hdv->hv", K, decayed)
            after = decayed + np.einsum("hd,h,hv->hdv", K, bt, miss)
            d = D[b] + scale * np.einsum("hd,hv->hdv", Q, dO[t, b])
            dq[t, b] = (scale * np.einsum("hdv,hv->hd", after, dO[t, b])).reshape(key_heads, group, -1).sum(1)
            du = np.einsum("hd,hdv->hv", K, d)
            dk[t, b] = (np.einsum("hdv,h,hv->hd", d, bt, miss) - np.einsum("h,hdv,hv->hd", bt, decayed, du)).reshape(key_heads, group, -1).sum(1)
            db[t, b] = (du * miss).sum(1)
            dv[t, b] = bt[:, None] * du
            ddecayed = d - np.einsum("h,hd,hv->hdv", bt, K, du)
            dg[t, b] = (ddecayed * decayed).sum((1, 2))
            if sizes is not None:
                sizes["dg"][t, b] = abs(ddecayed * decayed).sum((1, 2))
                sizes["dbeta"][t, b] = np.linalg.norm(du, axis=1) * np.linalg.norm(miss, axis=1)
            D[b] = a[:, None, None] * ddecayed
    return dq.reshape(T, B, -1), dk.reshape(T, B, -1), dv.reshape(T, B, -1), dg, db, D


# ---- scores of given tokens

def _existing(logits, allowed):
    l = np.array(logits, np.float64)
    if allowed is not None:
        l = np.where(np.broadcast_to(allowed, l.shape) != 0, l, -np.inf)
    return np.where(np.isnan(l), -np.inf, l)


def _log_shares(l):
    """log p of a row of which some tokens do not exist (minus infinity); infinite ones share all."""
    top = l.max()
    if top == -np.inf:
        return np.full(l.shape, -np.inf)
    with np.errstate(invalid="ignore"):
        d = np.where(l == top, 0.0, l - top)
    return d - np.log(np.exp(d).sum())


def logprobs_forward(logits, token=None, allowed=None, top_n=0):
    """Returns logprob, rank, entropy, top_token [M, top_n], top_logprob [M, top_n]."""
    l = _existing(logits, allowed)
    M, V = l.shape
    logprob, rank, entropy = np.zeros(M), np.full(M, -1), np.zeros(M)
    top_token, top_logprob = np.full((M, top_n), -1), np.full((M, top_n), -np.inf)
    for m in range(M):
        lp = _log_shares(l[m])
        p = np.exp(lp)
        entropy[m] = -(p[p > 0] * lp[p > 0]).sum()
        there = l[m] > -np.inf
        order = np.argsort(-l[m], kind="stable")[:there.sum()]
        n = min(top_n, len(order))
        top_token[m, :n], top_logprob[m, :n] = order[:n], lp[order[:n]]
        if token is not None and 0 <= token[m] < V:
            logprob[m] = lp[token[m]]
            mine, at = l[m, token[m]], np.arange(V)
            rank[m] = (there & ((l[m] > mine) | ((l[m] == mine) & (at < token[m])))).sum()
    return logprob, rank, entropy, top_token, top_logprob


def logprobs_backward(logits, token=None, allowed=None, dlogprob=None, dentropy=None):
    l = _existing(logits, allowed)
    M, V = l.shape
    out = np.zeros((M, V))
    for m in range(M):
        lp = _log_shares(l[m])
        p = np.exp(lp)
        if dlogprob is not None and 0 <= token[m] < V:
            out[m] -= float(dlogprob[m]) * p
            out[m, token[m]] += float(dlogprob[m])
        if dentropy is not None:
            plog = np.where(p > 0, p * np.where(p > 0, lp, 0.0), 0.0)
            out[m] -= float(dentropy[m]) * (plog - p * plog.sum())
        out[m, l[m] == -np.inf] = 0.0
    return out


# ---- distillation from a teacher's words

def distill(logits, top_token, top_logit, temperature, teacher_lse=None, dloss=None):
    """loss [M] and, for dloss, the gradient by the logits."""
    l = np.array(logits, np.float64)
    M, V = l.shape
    heat = float(temperature)
    loss, grad = np.zeros(M), np.zeros((M, V))
    for m in range(M):
        words, z = [], []
        for j, w in enumerate(top_token[m]):
            if 0 <= w < V and w not in words:
                words.append(int(w))
                z.append(float(top_logit[m, j]) / heat)
        words, z = np.array(words, int), np.array(z, np.float64)
        if teacher_lse is None:
            if not len(words):
                continue
            t = np.exp(z - z.max())
            t, t_rest = t / t.sum(), 0.0
        else:
            t = np.exp(z - float(teacher_lse[m]))
            t_rest = max(0.0, 1.0 - t.sum())
        log_s = _log_shares(l[m] / heat)
        outside = np.ones(V, bool)
        outside[words] = False
        if not outside.any():       # nobody is left to have what rounding leaves of 1
            t_rest = 0.0
        elif teacher_lse is not None and (l[m, outside] == -np.inf).all():
            size = (t[t > 0] * abs(z[t > 0])).sum() + abs(float(teacher_lse[m])) + 1
            t_rest = t_rest if t_rest > 2.0 ** -22 * size else 0.0
        with np.errstate(divide="ignore", invalid="ignore"):
            used = t > 0
            total = (t[used] * (np.log(t[used]) - log_s[words[used]])).sum()
            inner = _log_shares(log_s[outside]) if outside.any() else np.zeros(0)
            if t_rest > 0:
                best = log_s[outside].max() if outside.any() else -np.inf
                log_s_rest = best + np.log(np.exp(log_s[outside] - best).sum()) if best > -np.inf else -np.inf
                total += t_rest * (np.log(t_rest) - log_s_rest)
        loss[m] = heat * heat * total
        if dloss is not None:
            want = np.zeros(V)
            want[words] = t
            want[outside] = t_rest * np.exp(inner)
            grad[m] = float(dloss[m]) * heat * (np.exp(log_s) - want)
            if teacher_lse is None:
                grad[m, outside] = float(dloss[m]) * heat * np.exp(log_s[outside])
    return (loss, grad) if dloss is not None else loss
