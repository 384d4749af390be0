"""Which memory the recorded steps of the language model of examples/ hold: their own, whatever else runs on the stream."""
import pytest

from paper_1901_10997_amd import binding as B
from test_gpu_recurrent_lm import _tokens, lm  # noqa: F401

pytestmark = pytest.mark.gpu

# each entry that takes a workspace, and where among its arguments the address stands
ENTRIES = {"lstm_matmul_fp8": -3, "lstm_scan_forward": -3, "lstm_sample": -3}


def test_workspaces_of_a_step_are_its_writers(lm, monkeypatch):  # noqa: F811
    """The addresses that a step hands over are the same after larger calls on the stream, inside a tensor of the writer's, and not
    another writer's."""
    model = lm.RecurrentLm(500, 130, 2)
    logits, state = model.forward(_tokens(5, 3, 500), last_only=True)
    writers = [lm.Writer(model, logits.argmax(1), state) for _ in range(2)]
    seen = []
    for name, at in ENTRIES.items():
        def call(*a, entry=getattr(B, name), at=at):
            seen.append((a[at], a[at + 1]))
            entry(*a)
        monkeypatch.setattr(B, name, call)

    def addresses(writer):
        seen.clear()
        writer.step()
        assert len(seen) == 8               # three for each block, two behind them
        return list(seen)

    first = addresses(writers[0])
    lm._workspace(64 << 20)                 # what a larger call asks for
    assert addresses(writers[0]) == first
    other = addresses(writers[1])
    assert not {a for a, _ in first} & {a for a, _ in other}
    owned = [(t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()) for t in vars(writers[0]).values() if hasattr(t, "data_ptr")]
    assert all(any(lo <= a and a + n <= hi for lo, hi in owned) for a, n in first)


def test_recorded_steps_after_larger_calls(lm):  # noqa: F811
    """Replays between prompts and learning steps of other models draw what eager steps draw."""
    import torch
    model, other = lm.RecurrentLm(700, 200, 2), lm.RecurrentLm(300, 160, 1)
    logits, state = model.forward(_tokens(9, 4, 700), last_only=True)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(2)
    u = torch.rand((12, 4), generator=gen, device="cuda")
    eager = lm.Writer(model, logits.argmax(1), state, top_k=40)
    want = eager.write(u)
    writer = lm.Writer(model, logits.argmax(1), state, top_k=40)
    writer.record()
    out = []
    for i in range(4):
        out.append(writer.write(u[3 * i:3 * i + 3]))
        other.gradient(_tokens(60 * (i + 1), 2, 300), _tokens(60 * (i + 1), 2, 300, 5))
        lm._workspace((i + 2) << 20)
    assert torch.equal(torch.cat(out), want) and torch.equal(writer.state, eager.state)
