"""Handles on another device than the current one (no GPU: two devices are modelled)."""
import pytest
import torch


class Stream:
    def __init__(self, raw, index):
        self.cuda_stream, self.device_index, self.device = raw, index, torch.device("cuda", index)

    def wait_stream(self, other):
        assert other.device_index == self.device_index


@pytest.fixture
def machine(monkeypatch):
    """Two devices with a current stream each; calls: (current device, stream that the work goes to)."""
    from paper_2510_04206_amd import _binding as B

    class Machine:
        at, calls = 0, []
        current = [Stream(0, 0), Stream(0, 1)]
    m = Machine()
    m.calls = []
    index = lambda d: m.at if d is None else d if isinstance(d, int) else torch.device(d).index  # noqa: E731
    stream_of = lambda d=None: m.current[m.at if index(d) is None else index(d)]                 # noqa: E731
    empty = torch.empty

    class Device:
        def __init__(self, d):
            self.to = index(d)

        def __enter__(self):
            self.old, m.at = m.at, self.to

        def __exit__(self, *a):
            m.at = self.old

    class Using(Device):
        def __init__(self, s):
            self.to, self.s = s.device_index, s

        def __enter__(self):
            super().__enter__()
            self.was, m.current[self.to] = m.current[self.to], self.s

        def __exit__(self, *a):
            m.current[self.to] = self.was
            super().__exit__()

    monkeypatch.setattr(torch.cuda, "current_stream", stream_of)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: m.at)
    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(torch.cuda, "stream", Using)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda i: m.current[i].cuda_stream, raising=False)
    monkeypatch.setattr(torch, "empty", lambda *a, device=None, **k: empty(*a, **k))
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: None)
    for name in ("agrl_token_norm_fwd", "agrl_token_norm_bwd", "agrl_orthogonalize", "agrl_muon_step"):
        # (as the binding: no stream given is the current device's)
        monkeypatch.setattr(B, name, lambda *a: m.calls.append(
            (m.at, a[-1] if a[-1] is not None else m.current[m.at])))
    return m


def _handles(device):
    import paper_2510_04206_amd as P
    x = torch.zeros(8, 16)
    norm, back = (P.TokenNorm(8, 16, torch.float32, device=device) for _ in range(2))
    orth, muon = P.Orthogonalize(8, 16, device=device), P.MuonStep(8, 16, device=device)
    return [(norm, lambda s: norm.forward(x, stream=s)), (back, lambda s: back.backward(x, None, x, stream=s)),
            (orth, lambda s: orth(x, stream=s)), (muon, lambda s: muon(x, x, x, 0.1, stream=s))]


def test_the_work_goes_to_the_handles_device(machine):
    for op, call in _handles("cuda:1"):
        op.device = torch.device("cpu")              # (that of the model's tensors)
        machine.calls.clear()
        call(None)                                   # device 0 is current
        side = Stream(0x20, 1)
        call(side)
        machine.current[1] = other = Stream(0x30, 1)
        call(None)
        machine.current[1] = Stream(0, 1)
        assert [at for at, _ in machine.calls] == [1, 1, 1] and machine.at == 0
        assert [s.device_index for _, s in machine.calls] == [1, 1, 1]
        assert machine.calls[1][1] is side and machine.calls[2][1] is other


def test_a_device_without_a_number_is_the_current_one(machine):
    machine.at = 1
    handles = _handles("cuda")
    machine.at = 0
    for op, call in handles:
        assert op.device == torch.device("cuda", 1)
        op.device = torch.device("cpu")
        machine.calls.clear()
        call(None)
        assert machine.calls[0][0] == 1 and machine.calls[0][1].device_index == 1


def test_streams_and_tensors_of_another_device_are_refused(machine):
    for op, call in _handles("cuda:1"):
        with pytest.raises(ValueError, match="is on cpu"):
            call(None)
        op.device = torch.device("cpu")
        with pytest.raises(ValueError, match="stream"):
            call(Stream(0, 0))                       # the null stream's handle is that of device 1's, too
    assert not machine.calls
