"""The operators around the cells in numpy and 64 bits, from their formulas: gated linear recurrence and its gradient, RMS
norm and its gradient, e4m3 quantization, the product with block scales, and the draw of a token.  Test infrastructure."""
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
