"""Attention where its launches and their ways through change: which kernels serve a call, parts of a group's heads, and
the second pass over a tile whose weights ran out of range.  Bounds as in test_gpu_attention."""
import numpy as np
import pytest
import torch

from helpers import log
from test_gpu_attention import BF, F32, _check, _make, _np, _offsets, _ref, _run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 96, 128])
def test_only_the_queries_are_unaligned(d):
    """Forward by 16-byte copies of k and v, backward without."""
    import paper_2510_04206_amd as P
    T, H, G, off = 210, 4, 2, [0, 100, 200]
    log(f"attention unaligned q d={d}")
    q, k, v, do = _make(T, H, G, d, BF)
    flat = torch.zeros(T * H * d + 1, dtype=BF, device="cuda")
    qd = flat[1:].view(T, H, d)
    qd.copy_(q)
    op, st = P.PackedAttention(T, H, G, d, BF), _offsets(off)
    o, lse = op.forward(qd, k.cuda(), v.cuda(), st)
    got = dict(o=o, lse=lse, **dict(zip(("dq", "dk", "dv"), op.backward(qd, k.cuda(), v.cuda(), st, do.cuda()))))
    dead = np.zeros(T, bool)
    dead[200:] = True
    val, tol = _ref(_np(q), _np(k), _np(v), off, _np(do), d ** -0.5, BF)
    _check(got, val, tol, dead, d)


@pytest.mark.parametrize("H,G", [(8, 4), (4, 4)])
def test_key_tiles_that_fill_the_chip(H, G):
    """280 workgroups of key tiles: each takes all heads of its group (fewer are dealt to several)."""
    T = 70 * 128
    _run(T, H, G, 64, BF, [*range(0, T - 50, 97), T - 9])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
def test_weights_out_of_range(dtype, d):
    """Scores hundreds above the row's own, in some rows of a tile and over several tiles: those tiles are gone
    through again; the rows of a sequence of small scores in the same tile have the bits they have without."""
    import paper_2510_04206_amd as P
    T, off = 700, [0, 600, 700]
    log(f"attention out of range {dtype} {d}")
    q, k, v, do = _make(T, 2, 1, d, dtype)
    op, st = P.PackedAttention(T, 2, 1, d, dtype), _offsets(off)
    small = op.forward(q.cuda(), k.cuda(), v.cuda(), st)[0][600:].clone()
    k = k.float()
    k[20] *= 40
    k[333] *= 80
    k = k.to(dtype)
    o, lse = op.forward(q.cuda(), k.cuda(), v.cuda(), st)
    got = dict(o=o, lse=lse, **dict(zip(("dq", "dk", "dv"), op.backward(q.cuda(), k.cuda(), v.cuda(), st, do.cuda()))))
    val, tol = _ref(_np(q), _np(k), _np(v), off, _np(do), d ** -0.5, dtype)
    assert float(np.abs(val["lse"]).max()) > 100
    _check(got, val, tol, np.zeros(T, bool), (dtype, d))
    assert torch.equal(o[600:], small)
