"""The calls of one handle are ordered whatever streams they are made on (no GPU: streams are modelled).

A model stream knows which calls are over when its next work starts: those enqueued on it before, and,
after wait_stream, those of the other stream.  A handle's calls share its workspace and outputs, so
each must find the one before it among them.
"""
import itertools
import random

import pytest
import torch


class Stream:
    """What the handles use of a torch stream."""

    def __init__(self, raw, index=0):
        self.cuda_stream, self.device_index = raw, index
        self.device = torch.device("cuda", index)
        self.done, self.capturing = set(), False

    def wait_stream(self, other):
        assert self.capturing == other.capturing, "a capture waits for work outside it, or the reverse"
        self.done |= other.done


class Machine:
    """A current stream, and the calls that were launched: (name, stream, calls over at its start)."""

    def __init__(self, monkeypatch):
        from paper_2510_04206_amd import _binding as B
        from paper_2510_04206_amd import api
        self.streams = [Stream(raw) for raw in (0, 0x10, 0x20, 0x30)]
        self.current, self.calls, self.recorded = self.streams[0], [], set()
        empty, machine = torch.empty, self

        class Using:
            def __init__(self, s):
                self.s = s

            def __enter__(self):
                self.old, machine.current = machine.current, self.s

            def __exit__(self, *a):
                machine.current = self.old

        def launch(name):
            def call(*a):
                s = a[-1] if a[-1] is not None else machine.current
                machine.calls.append((name, s, set(s.done)))
                s.done.add(len(machine.calls) - 1)
            return call

        monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: self.current)
        monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
        monkeypatch.setattr(torch.cuda, "stream", Using)
        monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: self.current.capturing)
        monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda i: self.current.cuda_stream,
                            raising=False)
        monkeypatch.setattr(torch, "empty", lambda *a, device=None, **k: empty(*a, **k))
        monkeypatch.setattr(torch.Tensor, "record_stream",
                            lambda t, s: self.recorded.add((t.data_ptr(), s.cuda_stream)))
        for name in ("agrl_token_norm_fwd", "agrl_token_norm_bwd", "agrl_orthogonalize", "agrl_muon_step"):
            monkeypatch.setattr(B, name, launch(name))
        # (the model's tensors are the CPU's)
        monkeypatch.setattr(api._Owned, "_same_device", lambda *a: None, raising=False)


def _handle(kind):
    """A handle's call, taking the stream; and the buffers that its calls share."""
    import paper_2510_04206_amd as P
    x = torch.zeros(8, 16)
    if kind == "norm":
        op = P.TokenNorm(8, 16, torch.float32)
        turns = itertools.cycle((lambda s: op.forward(x, stream=s), lambda s: op.backward(x, None, x, stream=s)))
        return lambda s: next(turns)(s), (op.workspace, op.y, op.mean, op.rstd, op.dx, op.dweight, op.dbias)
    if kind == "orthogonalize":
        op = P.Orthogonalize(8, 16)
        return lambda s: op(x, stream=s), (op.workspace, op.out)
    op = P.MuonStep(8, 16)
    return lambda s: op(x, x, x, 0.1, stream=s), (op.workspace,)


KINDS = ["norm", "orthogonalize", "muon"]


@pytest.mark.parametrize("kind", KINDS)
def test_each_call_waits_for_the_one_before(kind, monkeypatch):
    m = Machine(monkeypatch)
    call, buffers = _handle(kind)
    rng = random.Random(1)
    # there and back, two side streams, then any order, by argument or as the current stream
    order = [0, 1, 0, 1, 1, 2, 1, 2, 0] + [rng.randrange(4) for _ in range(60)]
    for i, k in enumerate(order):
        if rng.random() < 0.5:
            m.current = m.streams[rng.randrange(4)]
            call(m.streams[k])
        else:
            m.current = m.streams[k]
            call(None)
        assert m.calls[i][1] is m.streams[k]
        if i:
            assert i - 1 in m.calls[i][2], f"call {i} on stream {k} does not wait for call {i - 1}"
    # the allocator knows of every stream but the one that the buffers were made on
    assert {(b.data_ptr(), s.cuda_stream) for b in buffers for s in m.streams[1:]} <= m.recorded


@pytest.mark.parametrize("kind", KINDS)
def test_a_capture_waits_for_nothing_outside_it(kind, monkeypatch):
    """Whoever captures has synchronised before; the stream that counts is the one that is used."""
    m = Machine(monkeypatch)
    call, _ = _handle(kind)
    call(None)
    m.streams[1].capturing = True
    call(m.streams[1])                       # captured, though the current stream is not
    m.current = m.streams[1]
    call(None)
    call(m.streams[2])                       # not captured, though the current stream is
    assert 0 in m.calls[3][2]
    m.streams[1].capturing = False
    m.current = m.streams[0]
    call(None)
    assert 3 in m.calls[4][2]


@pytest.mark.parametrize("kind", KINDS)
def test_a_stream_under_capture_cannot_be_waited_for(kind, monkeypatch):
    """The last call's stream is being captured: what it did before can no longer be waited for."""
    m = Machine(monkeypatch)
    call, _ = _handle(kind)
    call(m.streams[1])
    m.streams[1].capturing = True
    with pytest.raises(RuntimeError, match="captured"):
        call(m.streams[2])
    assert len(m.calls) == 1
