"""Device buffers for the tests of the operators around the cells: tensors with guard values in front, behind and between
rows, so that a write outside a result shows."""
import numpy as np

from paper_1901_10997_amd import binding as B

GUARD = -777.0
U32 = 2.0 ** -24            # half a step of fp32, relative
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
DTYPE = {"f32": B.LSTM_F32, "bf16": B.LSTM_BF16}


def torch_type(name):
    import torch
    return torch.bfloat16 if name == "bf16" else torch.float32


def rounded(a, name):
    """The values of `a` in that type, as float64."""
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, np.float32)).to(torch_type(name)).double().numpy()


class Buf:
    """[rows..., width] values inside a larger allocation: `off` elements in front of it, `pad` behind each row."""

    def __init__(self, shape, name="f32", pad=0, off=0, data=None, order=None):
        import torch
        self.shape, dt = tuple(shape), torch_type(name)
        *lead, width = self.shape
        order = list(range(len(lead))) if order is None else order       # leading dimensions from outer to inner
        strides, step = [0] * len(lead), width + pad
        for d in reversed(order):
            strides[d] = step
            step *= lead[d]
        self.flat = torch.full((off + step + 64,), GUARD, dtype=dt, device="cuda:0")
        self.t = self.flat.as_strided(self.shape, strides + [1], off)
        if data is not None:
            self.t.copy_(torch.from_numpy(np.ascontiguousarray(data, np.float32)).to(dt))
        self.strides = strides

    @property
    def ptr(self):
        return self.t.data_ptr()

    def get(self):
        """The values as float64, after a check that nothing around them was written."""
        import torch
        torch.cuda.synchronize()
        out = self.t.double().cpu().numpy()
        keep = self.flat.clone()
        keep.as_strided(self.t.shape, self.t.stride(), self.t.storage_offset()).fill_(GUARD)
        assert bool((keep == torch.tensor(GUARD, dtype=keep.dtype, device=keep.device)).all()), "written outside the result"
        return out


def dev(a):
    import torch
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to("cuda:0")


def ptr(t):
    return None if t is None else t.data_ptr()


def workspace(nbytes):
    import torch
    ws = torch.empty(max(nbytes, 16), dtype=torch.uint8, device="cuda:0")
    ws.fill_(0xA5)          # what it holds must not matter
    return ws


def close(got, want, tol, what=""):
    """Element by element: |got - want| <= tol; NaN and infinities in the same places."""
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    fine = np.isfinite(want)
    assert np.array_equal(fine, np.isfinite(got)), what
    assert np.array_equal(np.isnan(want), np.isnan(got)), what
    off = np.abs(np.where(fine, got - want, 0.0))
    tol = np.broadcast_to(tol, off.shape)
    worst = np.unravel_index(np.argmax(off - tol), off.shape) if off.size else None
    assert (off <= tol).all(), (what, worst, got[worst], want[worst], off[worst], tol[worst])
