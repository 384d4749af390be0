"""Log probabilities, ranks, entropies, top alternatives, the distillation loss and their gradients against the oracle.

Tolerances, in half steps u of fp32: a difference of two logits d is off by u |d|, exp by 4 u, sums are 64 bits wide, so the log of
a sum is off by the terms' 4 u + u times their mean |d|, and a result by half a step of its own.  exp of what is below 2^-126 is 0: off by less than
that times what it is multiplied with.  Gradients in bf16: half a step of bf16."""
import numpy as np
import pytest

from oracle import lm_ops as O
from paper_1901_10997_amd import binding as B
from tests.lm_ops_util import DTYPE, HALF, U32, Buf, close, dev, ptr, rounded, workspace

pytestmark = pytest.mark.gpu


def _i32(a):
    return dev(np.asarray(a, np.int32))


def _f32(a):
    return None if a is None else dev(np.asarray(a, np.float32))


def make(seed, M, V, name, spread=3.0):
    r = np.random.default_rng(seed)
    l = r.normal(size=(M, V)) * spread
    l[np.arange(M), r.integers(0, V, M)] += r.uniform(0, 12, M)
    token = r.integers(0, V, M)
    token = np.where(r.uniform(size=M) < 0.5, l.argmax(1), token)
    return rounded(l, name), token, r


def score(l, name, token, allowed=None, top_n=0, pad=0, off=0, stats=False, stream=None, allowed_ld=None):
    import torch
    M, V = l.shape
    logits = Buf((M, V), name, pad=pad, off=off, data=l)
    out = dict(logprob=torch.full((M + 1,), -777.0, device="cuda:0"), rank=torch.full((M + 1,), -777, dtype=torch.int32, device="cuda:0"),
               entropy=torch.full((M + 1,), -777.0, device="cuda:0"), stats=torch.full((M + 1, 4), -777.0, device="cuda:0") if stats else None,
               top_token=torch.full((M + 1, max(1, top_n)), -777, dtype=torch.int32, device="cuda:0"),
               top_logprob=torch.full((M + 1, max(1, top_n)), -777.0, device="cuda:0"))
    a = None if allowed is None else dev(np.ascontiguousarray(allowed, np.uint8))
    ws, tok = workspace(B.lstm_logprobs_workspace_bytes(M, V, top_n)), _i32(token)
    B.lstm_logprobs_forward(M, V, DTYPE[name], logits.ptr, V + pad, ptr(a), V if allowed_ld is None else allowed_ld, ptr(tok), ptr(out["logprob"]),
                            ptr(out["rank"]), ptr(out["entropy"]), ptr(out["stats"]), top_n, ptr(out["top_token"]), ptr(out["top_logprob"]), ptr(ws), ws.numel(),
                            stream)
    torch.cuda.synchronize()
    for key, t in out.items():
        if t is not None:
            assert bool((t[M:] == -777).all()), key         # nothing behind the last row
    return {k: None if t is None else t[:M] for k, t in out.items()}, logits, a


def check_score(l, token, got, allowed=None, top_n=0):
    lp, rank, h, top, top_lp = O.logprobs_forward(l, token, allowed, top_n)
    L = O._existing(l, allowed)
    span = np.array([np.max(x[x > -np.inf], initial=-1e9) - np.min(x[np.isfinite(x)], initial=1e9) if (x > -np.inf).any() else 0 for x in L])
    span = np.where(np.isfinite(span) & (span > 0), span, 0)
    mean = np.minimum(span, h + 1)                              # mean |d| is at most entropy + what the log of the sum adds
    host = {k: None if v is None else v.double().cpu().numpy() for k, v in got.items()}
    fin = lambda x: np.where(np.isfinite(x), abs(x), 0)         # noqa: E731
    close(host["logprob"], lp, U32 * (2 * fin(lp) + 6 + mean), "logprob")
    close(host["entropy"], h, U32 * (2 * h + 8 + 2 * mean + 4 * mean * h), "entropy")
    assert np.array_equal(host["rank"], rank)
    if top_n:
        assert np.array_equal(host["top_token"], top)
        close(host["top_logprob"], top_lp, U32 * (2 * fin(top_lp) + 6 + mean[:, None]), "top_logprob")


# one workgroup to a row and several; both sides of each segment's end
SIZES = [(1, 1), (3, 2), (5, 255), (4, 2048), (3, 2049), (2, 4097), (1, 10000), (2, 16384), (2, 16385), (1, 131072 + 3), (1100, 301), (700, 2500), (300, 20011), (1, 1 << 20)]


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("M,V", SIZES)
def test_scores(M, V, name):
    l, token, r = make(1, M, V, name)
    token[::7] = -1
    for top_n in (0, 1, 20) if M * V < 1 << 20 else (20,):
        got, _, _ = score(l, name, token, top_n=top_n)
        check_score(l, token, got, top_n=top_n)


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("M,V,pad,off", [(6, 37, 3, 1), (3, 5001, 5, 3), (40, 3000, 0, 7), (3, 40001, 1, 1)])
def test_masks_nan_infinities_and_padding(M, V, pad, off, name):
    l, token, r = make(2, M, V, name)
    allowed = (r.uniform(size=(M, V)) < 0.7).astype(np.uint8)
    l[allowed == 0] = r.choice([np.nan, np.inf, -np.inf, 1e30], size=(allowed == 0).sum())
    l[0, r.integers(0, V, 5)] = np.nan
    l[1, :3] = np.inf
    allowed[1, 1:3] = 1
    l[2, 1:] = -np.inf
    token[:3] = [int(np.flatnonzero(np.isnan(l[0]))[0]), 2, V - 1]
    if M > 4:
        allowed[3] = 0          # nothing is left of this row
        token[4] = V            # and this one has no token
        allowed[5] = 200        # any byte but 0
    l = rounded(l, name)
    got, _, _ = score(l, name, token, allowed, 64, pad=pad, off=off)
    check_score(l, token, got, allowed, 64)
    shared = allowed[-1:]
    got, _, _ = score(l, name, token, shared, 5, pad=pad, off=off, allowed_ld=0)
    check_score(l, token, got, np.broadcast_to(shared, l.shape), 5)


@pytest.mark.parametrize("kind", ["equal", "two", "falling", "rising", "zeros", "one_far", "bunched"])
@pytest.mark.parametrize("V", [100, 3000, 33000])
def test_order_of_hard_rows(V, kind):
    """Ties go to the lowest index; rows in which one thread or one segment holds all the largest."""
    at = np.arange(V)
    l = {"equal": np.zeros(V), "two": np.where(at % 3, 1.0, 2.0), "falling": -at / 8.0, "rising": at / 8.0, "zeros": np.where(at % 2, 0.0, -0.0),
         "one_far": np.where(at == V // 2, 300.0, -300.0 - at % 5), "bunched": np.where(at // 8 % 256 == 17, 50.0 + at % 8, 0.0)}[kind]
    l = np.stack([l, l[::-1]])
    for name in ("f32", "bf16"):
        v, token = rounded(l, name), [V // 3, V - 1]
        for top_n in (1, 7, 64):
            got, _, _ = score(v, name, token, top_n=top_n)
            check_score(v, token, got, top_n=top_n)


def test_fewer_tokens_than_alternatives():
    l = rounded(np.array([[3.0, 1.0, 2.0], [5.0, 5.0, 5.0]]), "f32")
    got, _, _ = score(l, "f32", [0, 2], top_n=64)
    check_score(l, [0, 2], got, top_n=64)


def score_gradient(l, name, token, dlp, dh, allowed=None, pad=0, off=0, in_place=False):
    got, logits, a = score(l, name, token, allowed, pad=pad, off=off, stats=True)
    M, V = l.shape
    out = logits if in_place else Buf((M, V), name, pad=pad, off=off)
    tok, w, e = _i32(token), _f32(dlp), _f32(dh)
    B.lstm_logprobs_backward(M, V, DTYPE[name], logits.ptr, V + pad, ptr(a), V, ptr(tok), ptr(got["stats"]), ptr(w), ptr(e), out.ptr, V + pad)
    return out.get()


def check_score_gradient(l, name, token, dlp, dh, got, allowed=None):
    want = O.logprobs_backward(l, token, allowed, dlp, dh)
    L = O._existing(l, allowed)
    tol = np.zeros(l.shape)
    for m in range(len(l)):
        lp = O._log_shares(L[m])
        p, lp = np.exp(lp), np.where(lp > -np.inf, lp, 0.0)
        h = -(p * lp).sum()
        given = dlp is not None and 0 <= token[m] < l.shape[1]
        w = abs(float(dlp[m])) if given else 0.0
        e = abs(float(dh[m])) if dh is not None else 0.0
        # p is off by (|d| + 8) u, the bracket by u times its own terms
        tol[m] = U32 * p * (w + e * (abs(lp) + h)) * (abs(lp) + h + 12) + U32 * p * e * 12 + (w + e * (abs(lp) + h)) * 2.0 ** -126
        if given:
            tol[m, token[m]] += 2 * U32 * w
    close(got, want, tol + HALF[name] * abs(want), "dlogits")


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("M,V,pad,off", [(3, 1, 0, 0), (5, 50, 3, 1), (40, 2500, 0, 0), (2, 8192, 0, 0), (2, 8195, 5, 3), (2, 40003, 0, 0)])
def test_score_gradient(M, V, pad, off, name):
    l, token, r = make(3, M, V, name)
    token[0] = -1
    dlp, dh = np.float32(r.normal(size=M)), np.float32(r.normal(size=M))
    for w, e in ((dlp, dh), (dlp, None), (None, dh), (None, None)):
        got = score_gradient(l, name, token, w, e, pad=pad, off=off)
        check_score_gradient(l, name, token, w, e, got)
    assert np.array_equal(score_gradient(l, name, token, dlp, dh, pad=pad, off=off, in_place=True), score_gradient(l, name, token, dlp, dh, pad=pad, off=off))


@pytest.mark.parametrize("name", ["f32", "bf16"])
def test_score_gradient_of_masked_rows(name):
    l, token, r = make(4, 6, 3001, name)
    allowed = (r.uniform(size=l.shape) < 0.7).astype(np.uint8)
    l[allowed == 0] = np.nan
    allowed[2] = 0
    l[3, 5:9] = np.inf
    allowed[3, 5:9] = 1
    token[3], token[4] = 6, int(np.flatnonzero(allowed[4] == 0)[0])
    dlp, dh = np.float32(r.normal(size=6)), np.float32(r.normal(size=6))
    got = score_gradient(l, name, token, dlp, dh, allowed)
    check_score_gradient(l, name, token, dlp, dh, got, allowed)


# ---- distillation

def distill(l, name, words, z, heat, lse, dloss=None, pad=0, off=0, in_place=False, list_pad=0):
    import torch
    (M, V), K = l.shape, words.shape[1]
    logits = Buf((M, V), name, pad=pad, off=off, data=l)
    wide = lambda a, t: dev(np.ascontiguousarray(np.pad(a, ((0, 0), (0, list_pad)), constant_values=7).astype(t)))     # noqa: E731
    w, zz, norm = wide(words, np.int32), wide(z, np.float32), _f32(lse)
    loss, stats = torch.full((M + 1,), -777.0, device="cuda:0"), torch.full((M + 1, 4), -777.0, device="cuda:0")
    ws = workspace(B.lstm_distill_workspace_bytes(M, V, K))
    args = (M, V, K, DTYPE[name], logits.ptr, V + pad, ptr(w), K + list_pad, ptr(zz), K + list_pad, ptr(norm), heat)
    B.lstm_distill_forward(*args, ptr(loss), ptr(stats), ptr(ws), ws.numel())
    torch.cuda.synchronize()
    assert float(loss[M]) == -777 and bool((stats[M] == -777).all())
    if dloss is None:
        return loss[:M].double().cpu().numpy(), None
    out = logits if in_place else Buf((M, V), name, pad=pad, off=off)
    d = _f32(dloss)
    B.lstm_distill_backward(*args, ptr(stats), ptr(d), out.ptr, V + pad)
    return loss[:M].double().cpu().numpy(), out.get()


def check_distill(l, name, words, z, heat, lse, dloss, got):
    heat = float(np.float32(heat))
    loss, grad = O.distill(l, words, z, heat, lse, dloss)
    tol_loss, tol = np.zeros(len(l)), np.zeros(l.shape)
    for m in range(len(l)):
        log_s = O._log_shares(np.asarray(l[m], np.float64) / heat)
        s, finite = np.exp(log_s), np.where(np.isfinite(log_s), abs(log_s), 0)
        mean = (s * finite).sum()
        used = [w for w in dict.fromkeys(int(w) for w in words[m]) if 0 <= w < l.shape[1]]
        outside = np.ones(l.shape[1], bool)
        outside[used] = False
        s_r = s[outside].sum()
        far = max([finite[w] for w in used], default=0.0) + (abs(np.log(s_r)) + 1 if s_r > 0 else 0) + mean
        tol_loss[m] = heat ** 2 * U32 * (2 * far + 12) + U32 * abs(loss[m]) if np.isfinite(loss[m]) else 0
        w = abs(float(dloss[m])) * heat
        want = s - grad[m] / (float(dloss[m]) * heat) if dloss[m] else np.zeros_like(s)      # t, or the word's part of t_r
        tol[m] = U32 * w * (s + abs(want)) * (finite + mean + 16) + 2 * w * 2.0 ** -126
    close(got[0], loss, tol_loss, "loss")
    if got[1] is not None:
        close(got[1], grad, tol + HALF[name] * abs(grad), "dlogits")


def teacher(l, r, K, heat, rest):
    z = l + r.normal(size=l.shape)
    words = np.argsort(-z, axis=1)[:, :K]
    words = r.permuted(words, axis=1)
    lse = np.float32(np.log(np.exp((z - 20) / heat).sum(1)) + 20 / heat).astype(np.float64) if rest else None
    return words, np.float32(np.take_along_axis(z, words, 1)).astype(np.float64), lse


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("rest", [True, False], ids=["rest", "list"])
@pytest.mark.parametrize("M,V,K,heat,pad,off", [(3, 1, 1, 1.0, 0, 0), (5, 40, 7, 2.0, 3, 1), (35, 2000, 16, 1.0, 0, 0), (2, 2049, 256, 0.5, 5, 3), (1, 30000, 64, 4.0, 0, 0),
                                                (1100, 300, 5, 1.5, 0, 0), (300, 20003, 33, 1.0, 1, 1), (2, 150000, 100, 1.0, 0, 0)])
def test_distill(M, V, K, heat, pad, off, rest, name):
    l, _, r = make(5, M, V, name)
    words, z, lse = teacher(l, r, K, heat, rest)
    dloss = np.float32(r.normal(size=M))
    check_distill(l, name, words, z, heat, lse, dloss, distill(l, name, words, z, heat, lse, dloss, pad, off, list_pad=2))
    a, b = (distill(l, name, words, z, heat, lse, dloss, pad, off, in_place=p)[1] for p in (True, False))
    assert np.array_equal(a, b)


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("rest", [True, False], ids=["rest", "list"])
def test_distill_of_unusual_lists(rest, name):
    """Words twice, words that are none, a row without a list, shares of 0, and a list that is the whole vocabulary."""
    l, _, r = make(6, 7, 9, name)
    words = r.integers(0, 9, (7, 9))
    words[0] = np.arange(9)
    words[1] = 4
    words[2] = [-1, 9, 1 << 30, -5, 3, 3, -(1 << 31), 8, 0]
    words[3] = -1
    z = np.float32(r.normal(size=(7, 9))).astype(np.float64)
    z[0, 3] = z[4, 1] = -np.inf
    lse = np.float32(np.log(np.exp(z).sum(1)) + 0.5).astype(np.float64) if rest else None
    if rest:
        lse[0] = np.float32(np.log(np.exp(z[0]).sum()) - 1e-3)      # a little more than 1: nothing is left for others
    dloss = np.float32(r.normal(size=7))
    check_distill(l, name, words, z, 1.0, lse, dloss, distill(l, name, words, z, 1.0, lse, dloss))


@pytest.mark.parametrize("name", ["f32", "bf16"])
def test_distill_of_far_logits(name):
    """A student that is sure against a teacher that is not: shares outside the list below the smallest number, and minus infinities."""
    l = np.zeros((4, 600))
    l[0, 5] = 300.0                 # words outside the list have e^-300
    l[1, 5], l[1, 7] = 90.0, 60.0
    l[2, 100:] = -np.inf
    l[3] = np.linspace(-200, 200, 600)
    l = rounded(l, name)
    words = np.array([[5, 6], [5, 7], [5, 6], [599, 598]])
    z = np.log(np.array([[0.5, 0.2]] * 4))
    z = np.float32(z).astype(np.float64)
    dloss = np.float32([1.0, -2.0, 0.5, 0.25])
    for lse in (np.zeros(4), None):
        check_distill(l, name, words, z, 1.0, lse, dloss, distill(l, name, words, z, 1.0, lse, dloss))


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("M,V", [(1, 10000), (600, 3000), (2, 70000)])
def test_nearly_sure_tokens(M, V, name):
    """log p, entropy and 1 - p of a token that leaves 1e-2 to 1e-12 to all others, to a few steps of fp32 of themselves."""
    r = np.random.default_rng(10)
    l = r.normal(size=(M, V))
    token = r.integers(0, V, M)
    l[np.arange(M), token] = np.log(V) + np.linspace(5, 28, M) if M > 1 else 24.0
    l = rounded(l, name)
    d = l - l.max(1, keepdims=True)
    others = np.where(np.arange(V) == token[:, None], 0, np.exp(d))
    rest = others.sum(1)
    log_p, entropy = -np.log1p(rest), np.log1p(rest) - (others * d).sum(1) / (1 + rest)
    got, _, _ = score(l, name, token, top_n=1)
    logprob, h, top_logprob = (got[k].double().cpu().numpy() for k in ("logprob", "entropy", "top_logprob"))
    # a weight 2^-t is off by its argument's rounding, t up to 52: half a step of it is 2^-19, times ln 2; the exponential's own and the sums' a few 2^-24; the sum over
    # thousands of others takes the mean of the first.  One of it all as a bound, and the result's own rounding.  The sum, 1 and the others, is in
    # 64 bits: behind the 1 come one addition in its thread, six in its wave, up to fifteen of waves, and as many again where segments are joined, each half a step: 2^-53
    sums = 2 * (1 + 6 + 15) * 2.0 ** -53
    tol = 2.0 ** -19 * np.log(2) + 8 * 2.0 ** -24
    assert (logprob <= 0).all() and (np.abs(logprob - log_p) <= tol * -log_p + sums).all() and (top_logprob[:, 0] == logprob).all()
    assert (np.abs(h - entropy) <= 2 * tol * entropy + sums).all()
    if name == "f32":
        grad = score_gradient(l, name, token, np.ones(M), np.zeros(M))
        grad = np.asarray(grad, np.float64)[np.arange(M), token]
        assert (np.abs(grad - rest / (1 + rest)) <= (tol + 8 * 2.0 ** -24) * rest + sums).all()


def test_nan_stays_in_its_row():
    l, _, r = make(7, 5, 3000, "f32")
    words, z, lse = teacher(l, r, 8, 1.0, True)
    clean = distill(l, "f32", words, z, 1.0, lse, np.ones(5))
    bad = l.copy()
    bad[1, 77] = np.nan
    bad[3, words[3, 2]] = np.nan
    bad_z = z.copy()
    bad_z[4, 0] = np.nan
    got = distill(bad, "f32", words, bad_z, 1.0, lse, np.ones(5))
    for m in (1, 3, 4):
        assert np.isnan(got[0][m]) and np.isnan(got[1][m]).any()
    for m in (0, 2):
        assert got[0][m] == clean[0][m] and np.array_equal(got[1][m], clean[1][m])


@pytest.mark.parametrize("V", [50, 40000])
def test_rows_and_lists_of_minus_infinities(V):
    l, _, r = make(9, 4, V, "f32")
    l[1] = -np.inf
    words, z, _ = teacher(l, r, 6, 1.0, False)
    z[2] = -np.inf
    loss, grad = distill(l, "f32", words, z, 1.0, None, np.ones(4))
    assert np.isnan(loss[1]) and np.isnan(grad[1]).all()
    assert np.isnan(loss[2]) and np.isnan(grad[2][words[2]]).all()
    assert np.isfinite(loss[[0, 3]]).all() and np.isfinite(grad[[0, 3]]).all()


def test_lists_shared_by_all_rows():
    """A row length of 0: one list for all."""
    import torch
    l, _, r = make(8, 4, 500, "f32")
    words, z, _ = teacher(l[:1], r, 6, 1.0, False)
    logits, w, zz = Buf((4, 500), "f32", data=l), _i32(words), _f32(z)
    loss, ws = torch.empty(4, device="cuda:0"), workspace(256)
    B.lstm_distill_forward(4, 500, 6, 0, logits.ptr, 500, ptr(w), 0, ptr(zz), 0, None, 1.0, ptr(loss), None, ptr(ws), 256)
    want, _ = distill(l, "f32", np.repeat(words, 4, 0), np.repeat(z, 4, 0), 1.0, None)
    assert np.array_equal(loss.double().cpu().numpy(), want)


def test_same_bits_again_on_streams_and_in_a_graph():
    import torch
    M, V, K = 20, 30000, 12
    l, token, r = make(9, M, V, "bf16")
    words, z, lse = teacher(l, r, K, 2.0, True)
    logits, tok, w, zz, norm, d = Buf((M, V), "bf16", data=l), _i32(token), _i32(words), _f32(z), _f32(lse), _f32(r.normal(size=M))

    def buffers():
        e = lambda *s, dtype=torch.float32: torch.empty(s, dtype=dtype, device="cuda:0")      # noqa: E731
        return dict(lp=e(M), rank=e(M, dtype=torch.int32), h=e(M), stats=e(M, 4), tt=e(M, 9, dtype=torch.int32), tl=e(M, 9), dl=e(M, V, dtype=torch.bfloat16),
                    loss=e(M), stats2=e(M, 4), dl2=e(M, V, dtype=torch.bfloat16), ws=workspace(B.lstm_logprobs_workspace_bytes(M, V, 9)),
                    ws2=workspace(B.lstm_distill_workspace_bytes(M, V, K)))

    def run(o):
        st = torch.cuda.current_stream().cuda_stream
        p = {k: ptr(v) for k, v in o.items()}
        B.lstm_logprobs_forward(M, V, 1, logits.ptr, V, None, 0, ptr(tok), p["lp"], p["rank"], p["h"], p["stats"], 9, p["tt"], p["tl"], p["ws"], o["ws"].numel(), st)
        B.lstm_logprobs_backward(M, V, 1, logits.ptr, V, None, 0, ptr(tok), p["stats"], ptr(d), ptr(d), p["dl"], V, st)
        rows = (M, V, K, 1, logits.ptr, V, ptr(w), K, ptr(zz), K, ptr(norm), 2.0)
        B.lstm_distill_forward(*rows, p["loss"], p["stats2"], p["ws2"], o["ws2"].numel(), st)
        B.lstm_distill_backward(*rows, p["stats2"], ptr(d), p["dl2"], V, st)

    def same(a, b):
        torch.cuda.synchronize()
        return all(bool((a[k] == b[k]).all()) for k in a if not k.startswith("ws"))

    first, other = buffers(), buffers()
    run(first)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        run(other)
    assert same(first, other)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        run(other)
    for turn in range(3):
        logits.t.add_(torch.randn_like(logits.t))
        graph.replay()
        torch.cuda.synchronize()
        run(first)
        assert same(first, other)


def test_rows_further_than_32_bits_count():
    import torch
    M, V = 3, 5000
    l, token, r = make(10, M, V, "bf16")
    words, z, lse = teacher(l, r, 4, 1.0, True)
    ld = 2 ** 32 // (M - 1) + 64
    store = torch.empty(ld * (M - 1) + V, dtype=torch.bfloat16, device="cuda:0")
    far = store.as_strided((M, V), (ld, 1))
    far.copy_(torch.from_numpy(l).to(torch.bfloat16))
    lp, stats, ws = torch.empty(M, device="cuda:0"), torch.empty(M, 4, device="cuda:0"), workspace(1 << 20)
    dlp, tok = _f32(np.ones(M)), _i32(token)
    B.lstm_logprobs_forward(M, V, 1, far.data_ptr(), ld, None, 0, ptr(tok), ptr(lp), None, None, ptr(stats), 0, None, None, ptr(ws), ws.numel())
    want, _, _ = score(l, "bf16", token)
    assert bool((lp == want["logprob"]).all())
    loss, stats2, dloss = torch.empty(M, device="cuda:0"), torch.empty(M, 4, device="cuda:0"), _f32(np.ones(M))
    w, zz, norm = _i32(words), _f32(z), _f32(lse)
    rows = (M, V, 4, 1, far.data_ptr(), ld, ptr(w), 4, ptr(zz), 4, ptr(norm), 1.0)
    B.lstm_distill_forward(*rows, ptr(loss), ptr(stats2), ptr(ws), ws.numel())
    near_loss, near_grad = distill(l, "bf16", words, z, 1.0, lse, np.ones(M))
    torch.cuda.synchronize()
    assert np.array_equal(loss.double().cpu().numpy(), near_loss)
    B.lstm_distill_backward(*rows, ptr(stats2), ptr(dloss), far.data_ptr(), ld)
    torch.cuda.synchronize()
    assert np.array_equal(far.double().cpu().numpy(), near_grad)
    far.copy_(torch.from_numpy(l).to(torch.bfloat16))
    B.lstm_logprobs_backward(M, V, 1, far.data_ptr(), ld, None, 0, ptr(tok), ptr(stats), ptr(dlp), None, far.data_ptr(), ld)
    near = score_gradient(l, "bf16", token, np.ones(M), None)
    torch.cuda.synchronize()
    assert np.array_equal(far.double().cpu().numpy(), near)
