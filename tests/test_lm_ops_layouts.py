"""Which layouts of rows the recurrence takes as outputs: those whose rows share no element, in whatever order they lie (no GPU needed:
refusals come before anything reaches the device, and what is taken is told from them by its error code)."""
import os
import subprocess
import sys

import pytest

from paper_1901_10997_amd import binding as B

P, BIG = 0x10000, 1 << 40


def _overlap(T, b, t_stride, b_stride, width):
    seen = set()
    for t in range(T):
        for s in range(b):
            for k in range(width):
                at = t * t_stride + s * b_stride + k
                if at in seen:
                    return True
                seen.add(at)
    return False


def _forward(T, b, H, h_t, h_b):
    B.lstm_scan_forward(T, b, H, 0, 0, P, 64, 32, None, None, P, h_t, h_b, None, None, P, BIG)


def _backward(T, b, H, d_t, d_b):
    B.lstm_scan_backward(T, b, H, 0, 0, P, 64, 32, None, P, P, 64, 32, None, P, d_t, d_b, None, P, BIG)


@pytest.mark.parametrize("call,name", [(_forward, "rows of h overlap"), (_backward, "rows of dP overlap")])
@pytest.mark.parametrize("T,b,H,t,s", [(5, 2, 8, 1, 1), (2, 2, 8, 1, 1), (5, 3, 8, 2, 3), (9, 4, 8, 3, 2), (1000, 701, 3, 700, 699), (3, 2, 8, 1.25, 1.125)])
def test_rows_that_share_elements_are_refused(call, name, T, b, H, t, s):
    """Strides of at least a row each, so that only the two together show it.  (t, s: strides in rows.)"""
    width = H if call is _forward else 4 * H
    t, s = int(t * width), int(s * width)
    if T < 100:
        assert _overlap(T, b, t, s, width)
    with pytest.raises(B.LstmError) as e:
        call(T, b, H, t, s)
    assert e.value.code == B.LSTM_ERR_ARG and name in str(e.value)


# In a process of its own that sees no device: what is not refused goes on to a launch, which must not find one.
TAKEN = """
import sys
sys.path[:0] = [%r, %r]
from paper_1901_10997_amd import binding as B
import test_lm_ops_layouts as L
for width in (1, 2, 5):
    for T in (1, 2, 3, 6):
        for b in (1, 2, 3, 7):
            for t in range(0, 30):
                for s in range(0, 30):
                    least = (t < width and T > 1) or (s < width and b > 1)
                    for call, w, H in ((L._forward, width, width),) + (((L._backward, width, width // 4),) if width %% 4 == 0 else ()):
                        try:
                            call(T, b, H, t, s)
                            code = 0
                        except B.LstmError as e:
                            code = e.code
                        refused = code == B.LSTM_ERR_ARG
                        assert refused == (least or L._overlap(T, b, t, s, w)), (T, b, t, s, w, code)
for T, b, t, s in ((1 << 20, 15, 1 << 40, 8), (3, 2, 1 << 40, 1 << 39), (15, 1 << 16, 8, 1 << 40), (2, 2, 8, 1 << 40)):
    try:
        L._forward(T, b, 8, t, s)
    except B.LstmError as e:
        assert e.code != B.LSTM_ERR_ARG, (T, b, t, s, str(e))
print("done")
"""


def test_every_layout_of_rows_apart_is_taken():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", TAKEN % (root, os.path.join(root, "tests"))], capture_output=True, text=True, timeout=300,
                       env=dict(os.environ, HIP_VISIBLE_DEVICES="-1"))
    assert r.returncode == 0 and r.stdout.split() == ["done"], r.stderr[-2000:]
