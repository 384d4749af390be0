"""Refusals of the operators around the cells: every bad argument is an error code with a text before anything reaches the
device (no GPU needed: the addresses are never used)."""
import pytest

from paper_1901_10997_amd import binding as B

P = 0x10000         # an address that is aligned to everything
BIG = 1 << 40


def _scan(**kw):
    a = dict(T=5, Bn=2, H=8, dtype=0, reverse=0, P=P, P_t=64, P_b=32, lengths=None, c0=None, h=P, h_t=16, h_b=8, cT=None, states=None, ws=P, ws_bytes=BIG)
    a.update(kw)
    B.lstm_scan_forward(a["T"], a["Bn"], a["H"], a["dtype"], a["reverse"], a["P"], a["P_t"], a["P_b"], a["lengths"], a["c0"], a["h"], a["h_t"], a["h_b"],
                        a["cT"], a["states"], a["ws"], a["ws_bytes"])


def _scan_back(**kw):
    a = dict(T=5, Bn=2, H=8, dtype=0, reverse=0, P=P, P_t=64, P_b=32, lengths=None, states=P, dh=P, dh_t=16, dh_b=8, dcT=None, dP=P, dP_t=64, dP_b=32, dc0=None,
             ws=P, ws_bytes=BIG)
    a.update(kw)
    B.lstm_scan_backward(a["T"], a["Bn"], a["H"], a["dtype"], a["reverse"], a["P"], a["P_t"], a["P_b"], a["lengths"], a["states"], a["dh"], a["dh_t"], a["dh_b"],
                         a["dcT"], a["dP"], a["dP_t"], a["dP_b"], a["dc0"], a["ws"], a["ws_bytes"])


def _norm(**kw):
    a = dict(M=3, N=130, dtype=1, x=P, x_ld=130, r=P, r_ld=130, w=None, eps=1e-5, s=P, s_ld=130, y=P, y_ld=130, y8=P, y8_ld=144, sc=P, sc_ld=2, rstd=None)
    a.update(kw)
    B.lstm_rmsnorm_forward(a["M"], a["N"], a["dtype"], a["x"], a["x_ld"], a["r"], a["r_ld"], a["w"], a["eps"], a["s"], a["s_ld"], a["y"], a["y_ld"], a["y8"],
                           a["y8_ld"], a["sc"], a["sc_ld"], a["rstd"])


def _norm_back(**kw):
    a = dict(M=3, N=130, dtype=1, s=P, s_ld=130, w=None, rstd=P, dy=P, dy_ld=130, d=None, d_ld=0, dx=P, dx_ld=130, dw=P, ws=P, ws_bytes=BIG)
    a.update(kw)
    B.lstm_rmsnorm_backward(a["M"], a["N"], a["dtype"], a["s"], a["s_ld"], a["w"], a["rstd"], a["dy"], a["dy_ld"], a["d"], a["d_ld"], a["dx"], a["dx_ld"],
                            a["dw"], a["ws"], a["ws_bytes"])


def _quantize(**kw):
    a = dict(M=3, N=130, dtype=0, rows=1, x=P, x_ld=130, q=P, q_ld=144, sc=P, sc_ld=2)
    a.update(kw)
    B.lstm_quantize_fp8(a["M"], a["N"], a["dtype"], a["rows"], a["x"], a["x_ld"], a["q"], a["q_ld"], a["sc"], a["sc_ld"])


def _product(**kw):
    a = dict(M=3, N=5, K=130, A=P, a_ld=144, asc=P, asc_ld=2, W=P, w_ld=144, wsc=P, wsc_ld=2, rows=128, bias=None, out=0, C=P, c_ld=5, ws=P, ws_bytes=BIG)
    a.update(kw)
    B.lstm_matmul_fp8(a["M"], a["N"], a["K"], a["A"], a["a_ld"], a["asc"], a["asc_ld"], a["W"], a["w_ld"], a["wsc"], a["wsc_ld"], a["rows"], a["bias"], a["out"],
                      a["C"], a["c_ld"], a["ws"], a["ws_bytes"])


def _sample(**kw):
    a = dict(M=3, V=50, dtype=0, l=P, ld=50, al=None, al_ld=0, te=None, tk=None, tp=None, mp=None, u=P, token=P, prob=None, kept=None, ws=P, ws_bytes=BIG)
    a.update(kw)
    B.lstm_sample(a["M"], a["V"], a["dtype"], a["l"], a["ld"], a["al"], a["al_ld"], a["te"], a["tk"], a["tp"], a["mp"], a["u"], a["token"], a["prob"], a["kept"],
                  a["ws"], a["ws_bytes"])


SCAN = [dict(T=-1), dict(Bn=-1), dict(H=0), dict(H=(1 << 26) + 1), dict(T=(1 << 30) + 1), dict(H=1 << 26, Bn=1 << 10), dict(dtype=2), dict(reverse=2), dict(P=None),
        dict(P=P + 2), dict(P=P + 1, dtype=1), dict(P_t=-1), dict(P_b=-32), dict(P_t=BIG * 2), dict(lengths=P + 1), dict(ws=None), dict(ws=P + 8)]
CALLS = [
    (_scan, SCAN + [dict(h=None), dict(h=P + 3), dict(h_t=7), dict(h_b=7), dict(c0=P + 2), dict(cT=P + 2), dict(states=P + 1)]),
    (_scan_back, SCAN + [dict(states=None), dict(dh=None), dict(dP=None), dict(dP_t=31), dict(dP_b=31), dict(dh_t=-1), dict(dh_b=-1), dict(dcT=P + 2), dict(dc0=P + 2),
                         dict(dP=P + 1), dict(dh=P + 2)]),
    (_norm, [dict(M=-1), dict(M=1 << 24), dict(N=0), dict(N=16385, x_ld=20000), dict(dtype=-1), dict(eps=-1.0), dict(eps=float("nan")), dict(x=None), dict(y8=None),
             dict(sc=None), dict(x_ld=129), dict(r_ld=129), dict(s_ld=0), dict(y_ld=-130), dict(x=P + 1), dict(r=P + 1), dict(w=P + 2), dict(y8=P + 8), dict(y8_ld=130),
             dict(y8_ld=128), dict(sc_ld=1), dict(sc=P + 2), dict(rstd=P + 1), dict(x_ld=BIG * 2)]),
    (_norm_back, [dict(M=-1), dict(N=0), dict(N=16385), dict(dtype=5), dict(s=None), dict(rstd=None), dict(dy=None), dict(dx=None), dict(s_ld=5), dict(dy_ld=5),
                  dict(dx_ld=5), dict(d=P, d_ld=5), dict(dw=P + 1), dict(ws=None), dict(ws=P + 4), dict(rstd=P + 2)]),
    (_quantize, [dict(M=-1), dict(N=-1), dict(M=1 << 26, N=1), dict(dtype=9), dict(rows=64), dict(rows=0), dict(x=None), dict(q=None), dict(sc=None), dict(x_ld=7),
                 dict(q=P + 4), dict(q_ld=130), dict(q_ld=128), dict(sc_ld=1), dict(sc=P + 1), dict(x=P + 2)]),
    (_product, [dict(M=-1), dict(N=-1), dict(K=-1), dict(M=1 << 24, N=1 << 24), dict(out=2), dict(rows=2), dict(A=None), dict(asc=None), dict(W=None), dict(wsc=None),
                dict(C=None), dict(A=P + 8), dict(W=P + 8), dict(a_ld=130), dict(w_ld=130), dict(a_ld=128), dict(w_ld=128), dict(asc_ld=1), dict(wsc_ld=1), dict(c_ld=4),
                dict(C=P + 2), dict(bias=P + 1), dict(ws=None), dict(ws=P + 4)]),
    (_sample, [dict(M=-1), dict(M=1 << 22), dict(V=0), dict(V=(1 << 20) + 1, ld=1 << 21), dict(dtype=3), dict(l=None), dict(u=None), dict(token=None), dict(ld=49),
               dict(l=P + 2), dict(al=P, al_ld=49), dict(te=P + 1), dict(tk=P + 2), dict(tp=P + 2), dict(mp=P + 3), dict(u=P + 1), dict(token=P + 2), dict(prob=P + 2),
               dict(kept=P + 2), dict(ws=None), dict(ws=P + 2)]),
]


@pytest.mark.parametrize("call,change", [(c, k) for c, all_ in CALLS for k in all_], ids=lambda v: v.__name__ if callable(v) else str(v))
def test_refused(call, change):
    with pytest.raises(B.LstmError) as e:
        call(**change)
    assert e.value.code == B.LSTM_ERR_ARG
    assert "lstm_" in str(e.value)


@pytest.mark.parametrize("call", [_scan, _scan_back, _norm_back, _product, _sample])
def test_small_workspace(call):
    with pytest.raises(B.LstmError) as e:
        call(ws_bytes=0)
    assert e.value.code == B.LSTM_ERR_NOMEM and "workspace" in str(e.value)


def test_workspace_of_what_is_refused_is_none():
    assert B.lstm_scan_workspace_bytes(-1, 1, 1) == B.lstm_scan_workspace_bytes(1, 1, 0) == 0
    assert B.lstm_rmsnorm_workspace_bytes(1, 16385) == 0
    assert B.lstm_matmul_fp8_workspace_bytes(1, -1, 1) == 0
    assert B.lstm_sample_workspace_bytes(1, 0) == 0


def test_nothing_to_do_is_no_error():
    """No rows: nothing is launched (there may be no device)."""
    _scan(Bn=0)
    _scan_back(Bn=0)
    _norm(M=0)
    _norm_back(M=0, dw=None)
    _quantize(M=0)
    _product(N=0)
    _sample(M=0)
