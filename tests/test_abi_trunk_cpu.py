"""Embedding, rotation and attention refuse bad arguments before any HIP call (no GPU needed)."""
import pytest
import torch

E_NULL, E_SHAPE, E_DTYPE, E_FLAGS, E_WS, E_HIP, E_UNSUP = -1, -2, -3, -4, -5, -6, -7
P = 1 << 12
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def L():
    from paper_2510_04206_amd import _binding
    return _binding.lib()


def _embed_fwd(L, **kw):
    a = dict(T=10, d=64, V=100, wt=0, dt=0, w=P, ids=P, m=None, scale=1.0, y=P, ldy=64)
    a.update(kw)
    return L.agrl_token_embed_fwd(*a.values(), None)


def _embed_bwd(L, **kw):
    a = dict(T=10, d=64, V=100, dt=0, ids=P, m=None, dy=P, ldy=64, scale=1.0, acc=0, ws=P, n=1 << 30, dw=P)
    a.update(kw)
    return L.agrl_token_embed_bwd(*a.values(), None)


@pytest.mark.parametrize("call", [_embed_fwd, _embed_bwd])
def test_embedding_common(L, call):
    for kw in (dict(T=-1), dict(T=1 << 31), dict(d=0), dict(d=(1 << 20) + 1), dict(V=0), dict(V=2 ** 31 - 1), dict(ldy=63)):
        assert call(L, **kw) == E_SHAPE, kw
    assert call(L, dt=2) == E_DTYPE
    for s in (INF, NAN):
        assert call(L, scale=s) == E_FLAGS
    assert call(L, ids=None) == E_NULL
    assert b"NULL" in L.agrl_last_error()


def test_embedding_forward(L):
    assert _embed_fwd(L, wt=9) == E_DTYPE
    assert _embed_fwd(L, w=None) == E_NULL and _embed_fwd(L, y=None) == E_NULL
    assert _embed_fwd(L, T=0, w=None, ids=None, y=None) == 0


def test_embedding_backward(L):
    assert _embed_bwd(L, acc=2) == E_FLAGS
    assert _embed_bwd(L, dy=None) == E_NULL and _embed_bwd(L, dw=None) == E_NULL
    f = L.agrl_token_embed_bwd_workspace_size
    need = f(10, 64, 100)
    assert need > 0 and _embed_bwd(L, n=need - 1) == E_WS and _embed_bwd(L, ws=None) == E_WS
    assert _embed_bwd(L, ws=P + 128) == E_UNSUP
    assert f(-1, 64, 100) == 0 and f(10, 0, 100) == 0 and f(10, 64, 0) == 0
    assert f(2 ** 31 - 1024, 1 << 20, 100) == 0                    # more workgroups than a grid has
    assert _embed_bwd(L, T=0, acc=1, ids=None, dy=None, dw=None) == 0


def _rotate(L, **kw):
    a = dict(T=10, h=4, d=64, rot=64, dt=0, x=P, ldx=256, hx=64, pos=P, base=1e4, inter=0, inv=0, y=2 * P, ldy=256,
             hy=64)
    a.update(kw)
    return L.agrl_rotate_heads(*a.values(), None)


def test_rotation(L):
    for kw in (dict(T=-1), dict(h=-1), dict(d=0), dict(rot=63), dict(rot=66), dict(rot=-2), dict(ldx=-1), dict(hx=-64),
               dict(ldy=255), dict(hy=63), dict(ldy=64, hy=0), dict(ldy=64, hy=576), dict(ldy=1 << 62, hy=1 << 62),
               dict(y=P, ldx=512), dict(y=P, hx=0)):
        assert _rotate(L, **kw) == E_SHAPE, kw
    assert _rotate(L, d=513, rot=2, ldx=4096, hx=513, ldy=4096, hy=513) == E_UNSUP
    assert _rotate(L, dt=2) == E_DTYPE
    for b in (0.0, -1.0, INF, NAN):
        assert _rotate(L, base=b) == E_FLAGS
    assert _rotate(L, inter=2) == E_FLAGS and _rotate(L, inv=-1) == E_FLAGS
    assert _rotate(L, x=None) == E_NULL and _rotate(L, y=None) == E_NULL
    assert _rotate(L, T=0, x=None, y=None) == 0 and _rotate(L, h=0) == 0
    assert _rotate(L, rot=0, y=P) == 0                             # nothing turns, nothing moves


def _heads(h, **kw):
    return [kw.get("p", P), kw.get("ld", h * 64), kw.get("hs", 64)]


def _fwd(L, T=10, n=1, H=4, G=2, d=64, dt=0, q={}, k={}, v={}, st=P, scale=1.0, o={}, lse=P):
    return L.agrl_attention_fwd(T, n, H, G, d, dt, *_heads(H, **q), *_heads(G, **k), *_heads(G, **v), st, scale,
                                *_heads(H, **o), lse, None)


def _bwd(L, T=10, n=1, H=4, G=2, d=64, dt=0, q={}, k={}, v={}, st=P, scale=1.0, o={}, lse=P, do={}, ws=P, size=1 << 30,
         dq={}, dk={}, dv={}):
    return L.agrl_attention_bwd(T, n, H, G, d, dt, *_heads(H, **q), *_heads(G, **k), *_heads(G, **v), st, scale,
                                *_heads(H, **o), lse, *_heads(H, **do), ws, size, *_heads(H, **dq),
                                *_heads(G, **dk), *_heads(G, **dv), None)


@pytest.mark.parametrize("call", [_fwd, _bwd])
def test_attention_common(L, call):
    for kw in (dict(T=-1), dict(T=(1 << 31) - 1), dict(n=-1), dict(n=2 ** 31 - 1), dict(H=0), dict(G=0), dict(H=3),
               dict(d=0), dict(T=1 << 30, H=256, G=1), dict(q=dict(ld=-1)), dict(k=dict(hs=-1)), dict(v=dict(ld=-5))):
        assert call(L, **kw) == E_SHAPE, kw
    assert call(L, d=129) == E_UNSUP
    assert call(L, dt=3) == E_DTYPE
    for s in (0.0, -1.0, INF, NAN):
        assert call(L, scale=s) == E_FLAGS
    for name in ("q", "k", "v", "o"):
        assert call(L, **{name: dict(p=None)}) == E_NULL
    assert call(L, st=None) == E_NULL
    assert call(L, T=0, q=dict(p=None), st=None) == 0


def test_attention_outputs(L):
    assert _fwd(L, o=dict(ld=255)) == E_SHAPE and _fwd(L, o=dict(hs=63)) == E_SHAPE
    for out in ("dq", "dk", "dv"):
        assert _bwd(L, **{out: dict(ld=100)}) == E_SHAPE
        assert _bwd(L, **{out: dict(p=None)}) == E_NULL
    assert _bwd(L, lse=None) == E_NULL and _bwd(L, do=dict(p=None)) == E_NULL
    f = L.agrl_attention_bwd_workspace_size
    need = f(10, 4, 2, 64, 0)
    assert need > 0 and _bwd(L, size=need - 1) == E_WS and _bwd(L, ws=None) == E_WS
    assert _bwd(L, ws=P + 8) == E_UNSUP
    assert f(0, 4, 2, 64, 0) == 0 and f(10, 4, 3, 64, 0) == 0 and f(10, 4, 2, 129, 0) == 0 and f(10, 4, 2, 64, 2) == 0


# ------------------------------------------------------------------ handles (two devices are modelled)
from test_handle_devices_cpu import Stream, machine  # noqa: E402,F401


@pytest.fixture
def modelled(machine, monkeypatch):                                               # noqa: F811
    from paper_2510_04206_amd import _binding as B
    for name in ("agrl_token_embed_fwd", "agrl_token_embed_bwd", "agrl_rotate_heads", "agrl_attention_fwd",
                 "agrl_attention_bwd"):
        monkeypatch.setattr(B, name, lambda *a: machine.calls.append(
            (machine.at, a[-1] if a[-1] is not None else machine.current[machine.at])))
    return machine


def _handles(device):
    import paper_2510_04206_amd as P
    ids, w, dy = torch.zeros(8, dtype=torch.int32), torch.zeros(20, 16), torch.zeros(8, 16)
    q, kv, st = torch.zeros(8, 4, 16), torch.zeros(8, 2, 16), torch.zeros(2, dtype=torch.int32)
    e1, e2 = (P.TokenEmbedding(8, 20, 16, torch.float32, device=device) for _ in range(2))
    rot = P.TokenRotation(8, 4, 16, torch.float32, device=device)
    a1, a2 = (P.PackedAttention(8, 4, 2, 16, torch.float32, device=device) for _ in range(2))
    return [(e1, lambda s: e1.forward(w, ids, stream=s)), (e2, lambda s: e2.backward(ids, dy, stream=s)),
            (rot, lambda s: rot(q, stream=s)), (a1, lambda s: a1.forward(q, kv, kv, st, stream=s)),
            (a2, lambda s: a2.backward(q, kv, kv, st, q, stream=s))]


def test_the_work_goes_to_the_handles_device(modelled):
    for op, call in _handles("cuda:1"):
        op.device = torch.device("cpu")              # (that of the model's tensors)
        modelled.calls.clear()
        call(None)                                   # device 0 is current
        side = Stream(0x20, 1)
        call(side)
        assert [at for at, _ in modelled.calls] == [1, 1] and modelled.at == 0
        assert modelled.calls[1][1] is side and modelled.calls[0][1].device_index == 1


def test_other_devices_are_refused(modelled):
    for op, call in _handles("cuda:1"):
        with pytest.raises(ValueError, match="is on cpu"):
            call(None)
        op.device = torch.device("cpu")
        with pytest.raises(ValueError, match="stream"):
            call(Stream(0, 0))
    assert not modelled.calls


def test_shapes_and_types_are_checked(modelled):
    import paper_2510_04206_amd as P
    z = lambda *s, dt=torch.float32: torch.zeros(*s, dtype=dt)                     # noqa: E731
    i32 = torch.int32
    e = P.TokenEmbedding(8, 20, 16, torch.float32, grads=False, device="cuda:0")
    e.device = torch.device("cpu")
    for bad in ((z(20, 15), z(8, dt=i32)), (z(20, 16), z(7, dt=i32))):
        with pytest.raises(ValueError):
            e.forward(*bad)
    for bad in ((z(20, 16, dt=torch.bfloat16), z(8, dt=i32)), (z(20, 16), z(8, dt=torch.int64))):
        with pytest.raises(TypeError):
            e.forward(*bad)
    with pytest.raises(ValueError, match="grads"):
        e.backward(z(8, dt=i32), z(8, 16))
    r = P.TokenRotation(8, 4, 16, torch.float32, output=False, device="cuda:0")
    r.device = torch.device("cpu")
    with pytest.raises(ValueError, match="out"):
        r(z(8, 4, 16))
    with pytest.raises(TypeError):
        r(z(8, 4, 16), z(8, dt=torch.int64), out=z(8, 4, 16))
    a = P.PackedAttention(8, 4, 2, 16, torch.float32, grads=False, device="cuda:0")
    a.device = torch.device("cpu")
    with pytest.raises(ValueError):
        a.forward(z(8, 4, 16), z(8, 4, 16), z(8, 2, 16), z(2, dt=i32))
    with pytest.raises(ValueError):
        a.forward(z(8, 4, 16), z(8, 2, 16), z(8, 2, 16), z(0, dt=i32))
    with pytest.raises(TypeError):
        a.forward(z(8, 4, 16), z(8, 2, 16), z(8, 2, 16), z(2, dt=torch.int64))
    with pytest.raises(ValueError, match="grads"):
        a.backward(z(8, 4, 16), z(8, 2, 16), z(8, 2, 16), z(2, dt=i32), z(8, 4, 16))
    assert not modelled.calls
