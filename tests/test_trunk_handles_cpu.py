"""Handles of embedding, rotation and attention on streams and devices, and what a backward is given (no GPU: modelled)."""
import itertools
import random

import pytest
import torch

from test_abi_trunk_cpu import modelled                                          # noqa: F401
from test_handle_devices_cpu import machine                                      # noqa: F401
from test_handle_streams_cpu import Machine

NAMES = ("agrl_token_embed_fwd", "agrl_token_embed_bwd", "agrl_rotate_heads", "agrl_attention_fwd", "agrl_attention_bwd")


def _handle(kind, device="cuda:0"):
    """A handle, its call taking the stream, and the buffers that its calls share."""
    import paper_2510_04206_amd as P
    F32 = torch.float32
    if kind == "embedding":
        ids, w, dy = torch.zeros(8, dtype=torch.int32), torch.zeros(20, 16), torch.zeros(8, 16)
        op = P.TokenEmbedding(8, 20, 16, F32, device=device)
        turns = itertools.cycle((lambda s: op.forward(w, ids, stream=s), lambda s: op.backward(ids, dy, stream=s)))
        return op, lambda s: next(turns)(s), (op.y, op.workspace, op.dweight)
    if kind == "rotation":
        op, x = P.TokenRotation(8, 4, 16, F32, device=device), torch.zeros(8, 4, 16)
        return op, lambda s: op(x, stream=s), (op.out,)
    q, kv, st = torch.zeros(8, 4, 16), torch.zeros(8, 2, 16), torch.zeros(2, dtype=torch.int32)
    op = P.PackedAttention(8, 4, 2, 16, F32, device=device)
    turns = itertools.cycle((lambda s: op.forward(q, kv, kv, st, stream=s), lambda s: op.backward(q, kv, kv, st, q, stream=s)))
    return op, lambda s: next(turns)(s), (op.o, op.lse, op.workspace, op.dqkv)


KINDS = ["embedding", "rotation", "attention"]


def _machine(monkeypatch):
    from paper_2510_04206_amd import _binding as B
    m = Machine(monkeypatch)

    def launch(*a):
        s = a[-1] if a[-1] is not None else m.current
        m.calls.append((None, s, set(s.done)))
        s.done.add(len(m.calls) - 1)
    for name in NAMES:
        monkeypatch.setattr(B, name, launch)
    return m


@pytest.mark.parametrize("kind", KINDS)
def test_each_call_waits_for_the_one_before(kind, monkeypatch):
    m = _machine(monkeypatch)
    _, call, buffers = _handle(kind)
    rng = random.Random(2)
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
    assert {(b.data_ptr(), s.cuda_stream) for b in buffers for s in m.streams[1:]} <= m.recorded


@pytest.mark.parametrize("kind", KINDS)
def test_captures(kind, monkeypatch):
    """A capture waits for nothing outside it; a stream under capture cannot be waited for."""
    m = _machine(monkeypatch)
    _, call, _ = _handle(kind)
    call(None)
    m.streams[1].capturing = True
    call(m.streams[1])
    call(m.streams[2])                       # behind the first call, not the captured one
    assert 0 in m.calls[2][2]
    m.streams[2].capturing = True
    with pytest.raises(RuntimeError, match="captured"):
        call(m.streams[3])
    assert len(m.calls) == 3


@pytest.mark.parametrize("kind", KINDS)
def test_a_device_without_a_number_is_the_current_one(kind, modelled):           # noqa: F811
    modelled.at = 1
    op, call, _ = _handle(kind, "cuda")
    modelled.at = 0
    assert op.device == torch.device("cuda", 1)
    op.device = torch.device("cpu")
    for _ in range(2):
        modelled.calls.clear()
        call(None)
        assert modelled.calls[0][0] == 1 and modelled.calls[0][1].device_index == 1 and modelled.at == 0


def test_a_backward_is_given_o_and_lse(modelled, monkeypatch):                   # noqa: F811
    import paper_2510_04206_amd as P
    from paper_2510_04206_amd import _binding as B
    seen = []
    monkeypatch.setattr(B, "agrl_attention_bwd", lambda *a: seen.append((modelled.at, a[11], a[12])))
    a = P.PackedAttention(8, 4, 2, 16, torch.float32, device="cuda:1")
    a.device = torch.device("cpu")
    q, kv, st = torch.zeros(8, 4, 16), torch.zeros(8, 2, 16), torch.zeros(2, dtype=torch.int32)
    o, lse = torch.zeros(8, 4, 16), torch.zeros(4, 8)
    a.backward(q, kv, kv, st, q)
    assert seen[-1][0] == 1 and seen[-1][1] is a.o and seen[-1][2] is a.lse
    a.backward(q, kv, kv, st, q, o=o, lse=lse)
    assert seen[-1][0] == 1 and seen[-1][1] is o and seen[-1][2] is lse
    for bad in (dict(o=o), dict(lse=lse), dict(o=torch.zeros(8, 2, 16), lse=lse), dict(o=o, lse=torch.zeros(8, 4))):
        with pytest.raises(ValueError):
            a.backward(q, kv, kv, st, q, **bad)
    with pytest.raises(TypeError):
        a.backward(q, kv, kv, st, q, o=o, lse=lse.double())
    assert len(seen) == 2
