"""Refusals of the delta rule, the scores and the distillation loss: every bad argument is an error code with a text before anything
reaches the device (no GPU needed: the addresses are never used)."""
import pytest

from paper_1901_10997_amd import binding as B

P = 0x10000         # an address that is aligned to everything
BIG = 1 << 40


def _inputs(a):
    return (a["T"], a["Bn"], a["H"], a["HK"], a["Dk"], a["Dv"], a["dtype"], a["q"], a["q_t"], a["q_b"], a["k"], a["k_t"], a["k_b"], a["v"], a["v_t"], a["v_b"],
            a["g"], a["g_t"], a["g_b"], a["beta"], a["beta_t"], a["beta_b"], a["lengths"], a["scale"])


DELTA = dict(T=5, Bn=2, H=4, HK=2, Dk=8, Dv=6, dtype=0, q=P, q_t=32, q_b=16, k=P, k_t=32, k_b=16, v=P, v_t=48, v_b=24, g=P, g_t=8, g_b=4, beta=P, beta_t=8, beta_b=4,
             lengths=None, scale=1.0, ws=P, ws_bytes=BIG)


def _delta(**kw):
    a = dict(DELTA, S0=None, o=P, o_t=48, o_b=24, ST=None, states=None)
    a.update(kw)
    B.lstm_delta_forward(*_inputs(a), a["S0"], a["o"], a["o_t"], a["o_b"], a["ST"], a["states"], a["ws"], a["ws_bytes"])


def _delta_back(**kw):
    a = dict(DELTA, states=P, do=P, do_t=48, do_b=24, dST=None, dq=P, dq_t=32, dq_b=16, dk=P, dk_t=32, dk_b=16, dv=P, dv_t=48, dv_b=24, dg=P, dg_t=8, dg_b=4, db=P, db_t=8,
             db_b=4, dS0=None)
    a.update(kw)
    B.lstm_delta_backward(*_inputs(a), a["states"], a["do"], a["do_t"], a["do_b"], a["dST"], a["dq"], a["dq_t"], a["dq_b"], a["dk"], a["dk_t"], a["dk_b"], a["dv"], a["dv_t"],
                          a["dv_b"], a["dg"], a["dg_t"], a["dg_b"], a["db"], a["db_t"], a["db_b"], a["dS0"], a["ws"], a["ws_bytes"])


def _score(**kw):
    a = dict(M=3, V=50, dtype=0, l=P, ld=50, al=None, al_ld=0, token=P, lp=P, rank=P, h=P, stats=None, n=3, tt=P, tl=P, ws=P, ws_bytes=BIG)
    a.update(kw)
    B.lstm_logprobs_forward(a["M"], a["V"], a["dtype"], a["l"], a["ld"], a["al"], a["al_ld"], a["token"], a["lp"], a["rank"], a["h"], a["stats"], a["n"], a["tt"], a["tl"],
                            a["ws"], a["ws_bytes"])


def _score_back(**kw):
    a = dict(M=3, V=50, dtype=0, l=P, ld=50, al=None, al_ld=0, token=P, stats=P, dlp=P, dh=None, dl=P, dl_ld=50)
    a.update(kw)
    B.lstm_logprobs_backward(a["M"], a["V"], a["dtype"], a["l"], a["ld"], a["al"], a["al_ld"], a["token"], a["stats"], a["dlp"], a["dh"], a["dl"], a["dl_ld"])


def _distill(**kw):
    a = dict(M=3, V=50, K=4, dtype=0, l=P, ld=50, tt=P, tt_ld=4, tl=P, tl_ld=4, lse=None, heat=1.0, loss=P, stats=None, ws=P, ws_bytes=BIG)
    a.update(kw)
    B.lstm_distill_forward(a["M"], a["V"], a["K"], a["dtype"], a["l"], a["ld"], a["tt"], a["tt_ld"], a["tl"], a["tl_ld"], a["lse"], a["heat"], a["loss"], a["stats"], a["ws"],
                           a["ws_bytes"])


def _distill_back(**kw):
    a = dict(M=3, V=50, K=4, dtype=0, l=P, ld=50, tt=P, tt_ld=4, tl=P, tl_ld=4, lse=None, heat=1.0, stats=P, dloss=P, dl=P, dl_ld=50)
    a.update(kw)
    B.lstm_distill_backward(a["M"], a["V"], a["K"], a["dtype"], a["l"], a["ld"], a["tt"], a["tt_ld"], a["tl"], a["tl_ld"], a["lse"], a["heat"], a["stats"], a["dloss"], a["dl"],
                            a["dl_ld"])


INPUTS = [dict(T=-1), dict(T=(1 << 30) + 1), dict(Bn=-1), dict(Bn=(1 << 24) + 1), dict(H=0), dict(HK=0), dict(H=5), dict(H=2, HK=4), dict(H=1 << 17, HK=1 << 17), dict(Dk=0),
          dict(Dk=257), dict(Dv=0), dict(Dv=(1 << 16) + 1), dict(Bn=1 << 20, H=64), dict(T=1 << 29, Bn=4), dict(Bn=1 << 10, H=1 << 8, Dv=1 << 12), dict(dtype=2),
          dict(scale=float("nan")), dict(scale=float("inf")), dict(q=None), dict(k=None), dict(v=None), dict(beta=None), dict(q=P + 2), dict(k=P + 1, dtype=1),
          dict(v=P + 1), dict(g=P + 2), dict(beta=P + 2), dict(q_t=-1), dict(k_b=-16), dict(v_t=BIG * 2), dict(g_t=-1), dict(beta_b=-4), dict(lengths=P + 2), dict(ws=None),
          dict(ws=P + 8)]
ROWS = [dict(M=-1), dict(M=1 << 22), dict(V=0), dict(V=(1 << 20) + 1, ld=1 << 21), dict(M=1 << 20, V=1 << 20, ld=1 << 20), dict(dtype=2), dict(l=None), dict(ld=49), dict(l=P + 2),
        dict(l=P + 1, dtype=1)]
LISTS = [dict(K=0), dict(K=257), dict(tt=None), dict(tl=None), dict(tt=P + 2), dict(tl=P + 1), dict(tt_ld=-4), dict(tl_ld=-1), dict(tl_ld=BIG * 2), dict(lse=P + 2), dict(heat=0.0),
         dict(heat=-1.0), dict(heat=float("nan")), dict(heat=float("inf")), dict(heat=1e-7)]
CALLS = [
    (_delta, INPUTS + [dict(o=None), dict(o=P + 2), dict(o_t=23), dict(o_b=23), dict(o_t=24, o_b=24), dict(S0=P + 2), dict(ST=P + 1), dict(states=P + 3)]),
    (_delta_back, INPUTS + [dict(states=None), dict(states=P + 2), dict(do=None), dict(do=P + 2), dict(do_t=-1), dict(dST=P + 2), dict(dq=None), dict(dk=None), dict(dv=None),
                            dict(db=None), dict(dq_t=15), dict(dk_b=15), dict(dv_t=24), dict(dg_t=3), dict(db_b=3), dict(dq=P + 2), dict(dg=P + 2), dict(db=P + 1), dict(dS0=P + 2)]),
    (_score, ROWS + [dict(n=-1), dict(n=65), dict(tt=None), dict(tl=None), dict(token=None), dict(token=None, lp=None), dict(token=P + 2), dict(lp=P + 1), dict(rank=P + 2),
                     dict(h=P + 2), dict(stats=P + 2), dict(tt=P + 2), dict(tl=P + 2), dict(al=P, al_ld=49), dict(ws=None), dict(ws=P + 8)]),
    (_score_back, ROWS + [dict(stats=None), dict(dl=None), dict(token=None), dict(dl_ld=49), dict(dl=P + 2), dict(dlp=P + 2), dict(dh=P + 2), dict(stats=P + 1), dict(al=P, al_ld=-1)]),
    (_distill, ROWS + LISTS + [dict(loss=P + 2), dict(stats=P + 2), dict(ws=None), dict(ws=P + 8)]),
    (_distill_back, ROWS + LISTS + [dict(stats=None), dict(dloss=None), dict(dl=None), dict(dl_ld=49), dict(dl=P + 2), dict(dloss=P + 2), dict(stats=P + 2)]),
]


@pytest.mark.parametrize("call,change", [(c, k) for c, all_ in CALLS for k in all_], ids=lambda v: v.__name__ if callable(v) else str(v))
def test_refused(call, change):
    with pytest.raises(B.LstmError) as e:
        call(**change)
    assert e.value.code == B.LSTM_ERR_ARG
    assert "lstm_" in str(e.value)


@pytest.mark.parametrize("call", [_delta, _delta_back, _score, _distill])
def test_small_workspace(call):
    with pytest.raises(B.LstmError) as e:
        call(ws_bytes=0)
    assert e.value.code == B.LSTM_ERR_NOMEM and "workspace" in str(e.value)


def test_workspace_of_what_is_refused_is_none():
    for bad in ((-1, 1, 1, 1, 1, 1), (1, 1, 3, 2, 1, 1), (1, 1, 1, 1, 257, 1), (1, 1, 1, 1, 1, 0)):
        assert B.lstm_delta_workspace_bytes(*bad) == B.lstm_delta_workspace_bytes(*bad, True) == 0
    assert B.lstm_logprobs_workspace_bytes(1, 0) == B.lstm_logprobs_workspace_bytes(1, 5, 65) == B.lstm_logprobs_workspace_bytes(-1, 5) == 0
    assert B.lstm_distill_workspace_bytes(1, 5, 0) == B.lstm_distill_workspace_bytes(1, 5, 257) == 0


def test_nothing_to_do_is_no_error():
    """No rows: nothing is launched (there may be no device)."""
    _delta(Bn=0)
    _delta_back(Bn=0)
    _score(M=0)
    _score_back(M=0)
    _distill(M=0)
    _distill_back(M=0)
