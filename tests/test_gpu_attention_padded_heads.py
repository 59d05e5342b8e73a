"""bf16 heads whose size is a multiple of 8 but not 64 or 128, which the pipelined kernels pad: masked values, layouts, packings,
and infinite elements of counted keys.  Bounds as in test_gpu_attention."""
import numpy as np
import pytest
import torch

import test_gpu_attention as A
from helpers import log
from test_gpu_attention import BF, F32, _make, _np, _offsets, _ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("d", [8, 40, 72, 80, 96, 120])
def test_masked_values_reach_no_one(bad, d):
    A.test_masked_values_reach_no_one(bad, BF, d)


@pytest.mark.parametrize("layout", ["fused", "heads first", "odd", "repeated"])
@pytest.mark.parametrize("d", [80, 96])
def test_layouts(layout, d):
    A._run(190, 4, 2, d, BF, [0, 60, 188], layout)


@pytest.mark.parametrize("name", A.PACKINGS)
@pytest.mark.parametrize("d", [72, 80, 96])
def test_packings(name, d):
    T, off = A.PACKINGS[name]
    A._run(T, 4, 2, d, BF, off)


@pytest.mark.parametrize("dtype,d", [(BF, 64), (BF, 72), (BF, 80), (BF, 96), (BF, 120), (BF, 128), (BF, 50), (F32, 80), (F32, 128)])
@pytest.mark.parametrize("at", [5, 70, 199])
def test_a_key_of_score_minus_infinity(dtype, d, at):
    """An element of a key is -inf where every query's is positive: the key's scores are -inf, its weights 0, its gradients 0;
    dq's column of that element is 0 times infinite in the rows that count the key, its others as without the key."""
    import paper_2510_04206_amd as P
    T, H, G, off = 200, 4, 2, [0, 120, 200]
    log(f"attention key of -inf at {at} {dtype} {d}")
    q, k, v, do = _make(T, H, G, d, dtype)
    q[..., d - 1] = 2.0
    # the values: the same key with an element that leaves its weights exactly 0 in 64 bits; the bounds: a key of scores -40,
    # whose weights (e^-40) and roundings (40 (d + 8) u) leave those of the other keys as they are
    none, low = k.clone(), k.clone()
    none[at, :, d - 1] = -2.0 ** 20
    low[at] = 0
    low[at, :, d - 1] = -40 / (2 * d ** -0.5)
    k[at, :, d - 1] = -float("inf")
    op, st = P.PackedAttention(T, H, G, d, dtype), _offsets(off)
    o, lse = op.forward(q.cuda(), k.cuda(), v.cuda(), st)
    dq, dk, dv = op.backward(q.cuda(), k.cuda(), v.cuda(), st, do.cuda())
    val, _ = _ref(_np(q), _np(none), _np(v), off, _np(do), d ** -0.5, dtype)
    _, tol = _ref(_np(q), _np(low), _np(v), off, _np(do), d ** -0.5, dtype)
    e = min(s for s in off[1:] if s > at)
    for name, t in dict(o=o, lse=lse, dk=dk, dv=dv, dq=dq).items():
        got, want = _np(t), val[name]
        if name == "dq":                                       # the column of the element, in the rows that count the key
            assert not np.isfinite(got[at:e, :, d - 1]).any()
            got, want = got.copy(), want.copy()
            got[at:e, :, d - 1] = want[at:e, :, d - 1] = 0
        assert np.isfinite(got).all(), name
        if name in ("dk", "dv"):
            assert not got[at].any(), name
        off_by = np.abs(got - want)
        assert (off_by <= tol[name] + 1e-15).all(), (name, float((off_by / (tol[name] + 1e-15)).max()))
