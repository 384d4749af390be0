"""The 64-bit oracle of the delta rule, the scores and the distillation loss against differences, hand-made cases and a block form."""
import numpy as np
import pytest

from oracle import lm_ops as O


def _delta_case(seed, T=5, B=2, heads=4, key_heads=2, Dk=3, Dv=2):
    r = np.random.default_rng(seed)
    k = r.normal(size=(T, B, key_heads, Dk))
    k /= np.linalg.norm(k, axis=-1, keepdims=True)
    return dict(q=r.normal(size=(T, B, key_heads * Dk)), k=k.reshape(T, B, -1), v=r.normal(size=(T, B, heads * Dv)), g=-r.exponential(size=(T, B, heads)),
                beta=r.uniform(size=(T, B, heads)), heads=heads, key_heads=key_heads, scale=0.7), r.normal(size=(B, heads, Dk, Dv)), r


def test_delta_rule_finds_what_it_stored():
    """beta = 1 and orthogonal keys without decay: a query equal to a key reads its value; a second value replaces the first."""
    q = np.eye(3)[[0, 0, 1, 0]].reshape(4, 1, 3)
    k = np.eye(3)[[0, 1, 0, 2]].reshape(4, 1, 3)
    v = np.array([[1.0, 2.0], [3.0, 4.0], [5.0, 6.0], [7.0, 8.0]]).reshape(4, 1, 2)
    o, S, _ = O.delta_forward(q, k, v, None, np.ones((4, 1, 1)), 1, 1, 1.0)
    assert np.array_equal(o[:, 0], [[1, 2], [1, 2], [3, 4], [5, 6]])
    assert np.array_equal(S[0, 0], [[5, 6], [3, 4], [7, 8]])


def test_delta_rule_is_its_matrix_form():
    c, S0, _ = _delta_case(0, heads=2, key_heads=2)
    o, S, _ = O.delta_forward(**c, S0=S0)
    T, B = c["beta"].shape[:2]
    for b in range(B):
        for h in range(2):
            M = S0[b, h]
            for t in range(T):
                k, q, v = (c[n][t, b].reshape(2, -1)[h] for n in "kqv")
                M = np.exp(c["g"][t, b, h]) * (np.eye(3) - c["beta"][t, b, h] * np.outer(k, k)) @ M + c["beta"][t, b, h] * np.outer(k, v)
                assert np.allclose(o[t, b].reshape(2, -1)[h], 0.7 * M.T @ q, atol=1e-13)
            assert np.allclose(S[b, h], M, atol=1e-13)


@pytest.mark.parametrize("lengths", [None, [3, 0]])
def test_delta_gradient_is_that_of_differences(lengths):
    c, S0, r = _delta_case(1)
    dO, dST = r.normal(size=c["v"].shape), r.normal(size=S0.shape)

    def value():
        o, S, _ = O.delta_forward(**c, S0=S0, lengths=lengths)
        return (o * dO).sum() + (S * dST).sum()

    _, _, front = O.delta_forward(**c, S0=S0, lengths=lengths)
    got = dict(zip(("q", "k", "v", "g", "beta", "S0"), O.delta_backward(**c, front=front, dO=dO, dST=dST, lengths=lengths)))
    for name, grad in got.items():
        x = S0 if name == "S0" else c[name]
        for at in r.choice(x.size, 12, replace=False):
            i, old = np.unravel_index(at, x.shape), x.flat[at]
            x[i] = old + 1e-5
            hi = value()
            x[i] = old - 1e-5
            lo = value()
            x[i] = old
            assert abs((hi - lo) / 2e-5 - grad[i]) <= 1e-7 * max(1, abs(grad).max()), (name, i)


def test_scores_by_hand():
    l = np.log(np.array([[4.0, 2.0, 2.0, 8.0]]))
    lp, rank, h, top, top_lp = O.logprobs_forward(l, [2], None, 5)
    p = np.array([4, 2, 2, 8]) / 16
    assert np.allclose(lp, np.log(2 / 16)) and rank[0] == 3 and np.allclose(h, -(p * np.log(p)).sum())
    assert list(top[0]) == [3, 0, 1, 2, -1] and np.allclose(np.exp(top_lp[0]), [0.5, 0.25, 0.125, 0.125, 0])
    lp, rank, h, _, _ = O.logprobs_forward(np.array([[np.nan, 1, 2], [-np.inf] * 3, [np.inf, 0, np.inf]]), [0, 1, 2], None)
    assert lp[0] == -np.inf and rank[0] == 2 and lp[1] == -np.inf and rank[1] == 0 and h[1] == 0
    assert np.isclose(lp[2], -np.log(2)) and rank[2] == 1 and np.isclose(h[2], np.log(2))


def test_score_gradient_is_that_of_differences():
    r = np.random.default_rng(2)
    l, token, allowed = r.normal(size=(3, 7)), [2, -1, 5], (r.uniform(size=(3, 7)) < 0.8).astype(np.uint8)
    allowed[0, 2] = 1
    dlp, dh = r.normal(size=3), r.normal(size=3)

    def value(x):
        lp, _, h, _, _ = O.logprobs_forward(x, token, allowed)
        return (dlp * np.where(np.isfinite(lp), lp, 0)).sum() + (dh * h).sum()

    allowed[2, 5] = 1
    grad = O.logprobs_backward(l, token, allowed, dlp, dh)
    for i in np.ndindex(l.shape):
        e = np.zeros(l.shape)
        e[i] = 1e-6
        assert abs((value(l + e) - value(l - e)) / 2e-6 - grad[i]) < 1e-8


@pytest.mark.parametrize("rest", [False, True])
def test_distill_gradient_is_that_of_differences(rest):
    r = np.random.default_rng(3)
    l, z = r.normal(size=(3, 8)), r.normal(size=(3, 4))
    words = np.array([[1, 5, 2, 1], [7, -1, 0, 8], [-1, -1, 9, -1]])
    lse = np.log(np.exp(z / 1.5).sum(1) * 1.4) if rest else None
    w = r.normal(size=3)
    loss, grad = O.distill(l, words, z, 1.5, lse, w)
    assert loss[2] == 0 and (grad[2] == 0).all() if not rest else abs(loss[2]) < 1e-15 and abs(grad[2]).max() < 1e-15
    for i in np.ndindex(l.shape):
        e = np.zeros(l.shape)
        e[i] = 1e-6
        d = (O.distill(l + e, words, z, 1.5, lse) - O.distill(l - e, words, z, 1.5, lse)) / 2e-6
        assert abs((d * w).sum() - grad[i]) < 1e-8


def test_distill_of_the_teacher_itself_is_nothing():
    z = np.random.default_rng(4).normal(size=(2, 6)) * 3
    lse = np.log(np.exp(z / 2).sum(1))
    words = np.argsort(-z, axis=1)[:, :3]
    loss, grad = O.distill(z, words, np.take_along_axis(z, words, 1), 2.0, lse, np.ones(2))
    assert abs(loss).max() < 1e-14 and abs(grad).max() < 1e-14
