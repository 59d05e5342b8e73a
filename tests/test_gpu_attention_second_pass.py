"""The second pass over a tile of the pipelined forward: which rows it changes, and rows whose weights times v run out of range.
Bounds as in test_gpu_attention."""
import numpy as np
import pytest
import torch

from helpers import log
from test_gpu_attention import BF, F32, _check, _make, _np, _offsets, _ref

pytestmark = pytest.mark.gpu


def _above(T, H, G, d, dtype, powers, upto):
    """Inputs whose tokens before `upto` see their first key `powers` of 2 above their own scores."""
    q, k, v, do = _make(T, H, G, d, dtype)
    q, k = q.float(), k.float()
    q[:upto, :, 0] = 8.0
    k[:upto, :, 0] = 0.0
    k[0, :, 0] = powers / (8.0 * d ** -0.5 * 1.4426950408889634)
    return q.to(dtype), k.to(dtype), v, do


@pytest.mark.parametrize("powers", [40, 70, 80])
@pytest.mark.parametrize("bad", ["another sequence's v", "padding"])
@pytest.mark.parametrize("dtype,d", [(BF, 64), (BF, 80), (BF, 128), (F32, 128)])
def test_high_rows_keep_their_bits(powers, bad, dtype, d):
    """Rows whose largest score is many powers of 2 above their own, in a tile where another token is NaN."""
    import paper_2510_04206_amd as P
    T, H, G, off = 500, 2, 1, [0, 300, 480]
    log(f"attention {powers} powers above, {bad} {dtype} {d}")
    q, k, v, do = (t.cuda() for t in _above(T, H, G, d, dtype, powers, 300))
    op, st = P.PackedAttention(T, H, G, d, dtype, grads=False), _offsets(off)
    want = [t.clone() for t in op.forward(q, k, v, st)]
    val, tol = _ref(*(_np(t) for t in (q, k, v)), off, _np(do), d ** -0.5, dtype)
    dead = np.arange(T) >= 480
    _check(dict(o=want[0], lse=want[1]), val, tol, dead, (powers, d))
    v[320 if bad != "padding" else 490] = float("nan")
    got = op.forward(q, k, v, st)
    n = 320 if bad != "padding" else T
    assert torch.equal(got[0][:n], want[0][:n]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("powers,size", [(60, 2.0 ** 70), (90, 2.0 ** 60), (130, 2.0 ** 70), (5, 2.0 ** 90), (300, 2.0 ** 100)])
@pytest.mark.parametrize("dtype,d", [(BF, 64), (BF, 80), (BF, 128), (F32, 128)])
def test_large_values(powers, size, dtype, d):
    """Weights of many powers of 2 above a row's own times large finite elements of v: o lies between v's elements."""
    import paper_2510_04206_amd as P
    T, H, G, off = 400, 2, 1, [0, 300, 400]
    log(f"attention {powers} powers above, v around {size} {dtype} {d}")
    q, k, v, do = _above(T, H, G, d, dtype, powers, 300)
    v = (v.float() * size).to(dtype)
    op = P.PackedAttention(T, H, G, d, dtype, grads=False)
    o, lse = op.forward(q.cuda(), k.cuda(), v.cuda(), _offsets(off))
    val, tol = _ref(*(_np(t) for t in (q, k, v)), off, _np(do), d ** -0.5, dtype)
    _check(dict(o=o, lse=lse), val, tol, np.zeros(T, bool), (powers, size, d))
