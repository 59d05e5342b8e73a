"""The norm entry points refuse bad arguments before any HIP call (no GPU needed)."""
import pytest

E_NULL, E_SHAPE, E_DTYPE, E_FLAGS, E_WS, E_HIP, E_UNSUP = -1, -2, -3, -4, -5, -6, -7
P = 1 << 12


@pytest.fixture(scope="module")
def L():
    from paper_2510_04206_amd import _binding
    return _binding.lib()


def _fwd(L, **kw):
    a = dict(T=10, d=64, kind=0, dt=0, wt=1, x=P, ldx=64, w=P, b=P, m=None, eps=1e-5, y=P, ldy=64,
             mean=P, rstd=P)
    a.update(kw)
    return L.agrl_token_norm_fwd(*a.values(), None)


def _bwd(L, **kw):
    a = dict(T=10, d=64, kind=0, dt=0, wt=1, yt=1, x=P, ldx=64, w=P, m=None, dy=P, lddy=64, mean=P,
             rstd=P, acc=0, ws=P, n=1 << 20, dx=P, lddx=64, dw=P, db=P)
    a.update(kw)
    return L.agrl_token_norm_bwd(*a.values(), None)


@pytest.mark.parametrize("call", [_fwd, _bwd])
def test_common_refusals(L, call):
    assert call(L, T=-1) == E_SHAPE
    assert call(L, T=(1 << 40) + 1) == E_SHAPE
    assert call(L, d=0) == E_SHAPE
    assert call(L, ldx=63) == E_SHAPE
    assert call(L, dt=2) == E_DTYPE
    assert call(L, wt=-1) == E_DTYPE
    assert call(L, kind=2) == E_FLAGS
    assert call(L, d=16385, **{k: 16385 for k in ("ldx", "ldy" if call is _fwd else "lddy")}) == E_UNSUP
    assert call(L, x=None) == E_NULL
    assert b"NULL" in L.agrl_last_error()


def test_forward_refusals(L):
    assert _fwd(L, ldy=10) == E_SHAPE
    assert _fwd(L, y=None) == E_NULL
    for eps in (-1e-9, float("nan"), float("inf")):
        assert _fwd(L, eps=eps) == E_FLAGS
    assert _fwd(L, T=0, x=None, y=None) == 0          # nothing to do, nothing read


def test_backward_refusals(L):
    assert _bwd(L, yt=5) == E_DTYPE
    assert _bwd(L, lddy=63) == E_SHAPE
    assert _bwd(L, lddx=63) == E_SHAPE
    assert _bwd(L, acc=2) == E_FLAGS
    for k in ("dy", "dx", "rstd", "mean"):
        assert _bwd(L, **{k: None}) == E_NULL
    need = L.agrl_token_norm_bwd_workspace_size(10, 64)
    assert need > 0
    assert _bwd(L, n=need - 1) == E_WS
    assert _bwd(L, ws=None) == E_WS
    assert _bwd(L, ws=P + 2) == E_UNSUP
    f = L.agrl_token_norm_bwd_workspace_size
    assert f(0, 64) == 0 and f(10, 0) == 0 and f(10, 16385) == 0 and f(-1, 64) == 0
    assert f(1 << 20, 5120) <= 64 << 20               # bounded however many rows
