"""The orthogonalisation entry points refuse bad arguments before any HIP call (no GPU needed)."""
import ctypes

import pytest

E_NULL, E_SHAPE, E_DTYPE, E_FLAGS, E_WS, E_HIP, E_UNSUP = -1, -2, -3, -4, -5, -6, -7
P = 1 << 12


@pytest.fixture(scope="module")
def L():
    from paper_2510_04206_amd import _binding
    return _binding.lib()


def _orth(L, **kw):
    a = dict(batch=1, m=8, n=16, dt=1, g=P, ldg=16, sg=0, ot=0, ns=None, ws=P, n_ws=1 << 24, o=P,
             ldo=16, so=0)
    a.update(kw)
    return L.agrl_orthogonalize(*a.values(), None)


def _muon(L, **kw):
    a = dict(batch=1, m=8, n=16, dt=1, g=P, ldg=16, sg=0, pt=0, p=P, ldp=16, sp=0, mom=P, lr=0.1,
             mu=0.9, nest=1, wd=0.0, scale=0.0, ns=None, ws=P, n_ws=1 << 24)
    a.update(kw)
    return L.agrl_muon_step(*a.values(), None)


@pytest.mark.parametrize("call,ldo,so", [(_orth, "ldo", "so"), (_muon, "ldp", "sp")])
def test_common_refusals(L, call, ldo, so):
    from paper_2510_04206_amd._binding import agrl_ns_options as ns
    opt = lambda **k: ctypes.byref(ns(**k))                                       # noqa: E731
    for k in ("batch", "m", "n"):
        assert call(L, **{k: -1}) == E_SHAPE
        assert call(L, **{k: 0}, g=None, ws=None) == 0
    assert call(L, dt=3) == E_DTYPE
    assert call(L, ldg=15) == E_SHAPE
    assert call(L, **{ldo: 15}) == E_SHAPE
    assert call(L, batch=2, sg=-1, **{so: 128}) == E_SHAPE
    assert call(L, batch=2, sg=128, **{so: 127}) == E_SHAPE
    big = dict(ldg=1 << 21, **{ldo: 1 << 21})
    assert call(L, n=(1 << 20) + 1, **big) == E_SHAPE
    assert call(L, m=70000, n=70000, **big) == E_SHAPE
    assert call(L, g=None) == E_NULL
    assert call(L, ws=None) == E_WS
    assert call(L, ws=P + 128) == E_UNSUP
    assert call(L, ns=opt(steps=-1)) == E_FLAGS
    assert call(L, ns=opt(steps=101)) == E_FLAGS
    assert call(L, ns=opt(b=float("inf"))) == E_FLAGS
    assert call(L, ns=opt(eps=-1.0)) == E_FLAGS
    assert call(L, ns=opt(eps=float("nan"))) == E_FLAGS
    need = L.agrl_orthogonalize_workspace_size(1, 8, 16, 0)
    assert call(L, n_ws=need - 1) == E_WS
    assert b"workspace" in L.agrl_last_error()


def test_own_refusals(L):
    assert _orth(L, ot=2) == E_DTYPE
    assert _orth(L, o=None) == E_NULL
    assert _muon(L, pt=-1) == E_DTYPE
    assert _muon(L, p=None) == E_NULL
    assert _muon(L, mom=None) == E_NULL
    assert _muon(L, nest=2) == E_FLAGS
    for k in ("lr", "mu", "wd", "scale"):
        assert _muon(L, **{k: float("nan")}) == E_FLAGS
    assert _muon(L, scale=-1.0) == E_FLAGS


def test_workspace_size(L):
    f = L.agrl_orthogonalize_workspace_size
    assert f(0, 8, 16, 0) == 0 and f(1, 0, 16, 0) == 0 and f(1, 8, -1, 0) == 0 and f(1, 8, 16, 2) == 0
    assert f(1, (1 << 20) + 1, 4, 0) == 0 and f(65536, 8, 8, 0) == 0
    assert 0 < f(1, 200, 300, 0) < f(1, 200, 300, 1)         # fp32 results hold the products in two parts
    assert 0 < f(1, 100, 300, 0) <= f(1, 100, 300, 1)        # few rows: bf16 ones too
    assert f(1, 100, 300, 0) == f(1, 300, 100, 0)
    # a few planes of the matrix, not a multiple that grows
    assert f(1, 5120, 5120, 0) <= 14 * 5120 * 5120


def test_options_layout_matches_header(tmp_path):
    import os
    import shutil
    import subprocess
    from paper_2510_04206_amd._binding import agrl_ns_options as ns
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("gcc not found")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    names = [f[0] for f in ns._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "agrl.h"\nint main(void) {\n'
                   '  printf("%zu", sizeof(agrl_ns_options));\n' +
                   "".join(f'  printf(" %zu", offsetof(agrl_ns_options, {n}));\n' for n in names) +
                   "  return 0;\n}\n")
    exe = tmp_path / "layout"
    subprocess.run([gcc, "-I", os.path.join(root, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(v) for v in subprocess.run([str(exe)], capture_output=True, text=True,
                                          check=True).stdout.split()]
    assert got == [ctypes.sizeof(ns)] + [getattr(ns, n).offset for n in names]
