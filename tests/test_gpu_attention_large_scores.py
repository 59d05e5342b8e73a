"""Attention of finite inputs whose scores are so large that fp32 holds them to many units only.

Rows of one key each: the gaps between a row's scores are thousands of units or more, so one weight is 1 and the others 0 and
    o = v of that key, exactly;  lse = its score S, off by the product's (d + 8) u scale sum|q k| and 8 u |S|
    dv = the sum of do over the rows of the key: each weight is exactly 1 (S is formed the same way in each kernel, and is
         the lse where the sum is 1), so (n + r) of sum |do|, as for any weights
    dS = dP - D = 0 in exact arithmetic, two sums of d products of do and v: 2 (d + 8) u sum |do v|, rounded once more (1 + 2 r)
    dq, dk = 0, off by scale dS |k| and by scale sum dS |q|
with u = 2^-24 and r the type's half step.
"""
import numpy as np
import pytest
import torch

from helpers import log
from test_gpu_attention import BF, F32, HALF, U, _np, _offsets

pytestmark = pytest.mark.gpu


def _steps(n):
    """The n smallest bf16 numbers from 1 on: 2^-7 to 2^-8 of themselves apart."""
    return torch.from_numpy((np.arange(n, dtype=np.int32) + 0x3f80 << 16).view(np.float32).copy())


def _inputs(order, T, H, d, size, seed):
    """Keys c_j size w, queries a_n w, with c the first T bf16 numbers from 1 on in some order."""
    g = torch.Generator().manual_seed(seed)
    w = torch.randn(d, generator=g)
    c = _steps(T)
    if order == "falling":
        c = c.flip(0)
    elif order == "mixed":
        c = c[torch.randperm(T, generator=g)]
    q = (1 + torch.rand(T, H, 1, generator=g)) * w
    k = (size * c)[:, None, None] * w
    v, do = torch.randn(T, 1, d, generator=g), torch.randn(T, H, d, generator=g)
    return q, k, v, do


@pytest.mark.parametrize("order", ["rising", "falling", "mixed"])
@pytest.mark.parametrize("log2_score", [17, 24, 29, 31, 40, 90])
@pytest.mark.parametrize("dtype,d", [(BF, 64), (BF, 80), (BF, 128), (BF, 50), (F32, 64), (F32, 128)])
def test_rows_of_one_key(order, log2_score, dtype, d):
    import paper_2510_04206_amd as P
    T, H, off = 300, 2, [0, 150, 151, 299]
    log(f"attention scores 2^{log2_score} {order} {dtype} {d}")
    # half of the size in the keys, the rest in the scale where it has room
    scale = 2.0 ** min(60, log2_score // 2)
    size = 2.0 ** log2_score / (scale * d)
    q, k, v, do = (t.to(dtype) for t in _inputs(order, T, H, d, size, log2_score))
    op, st = P.PackedAttention(T, H, 1, d, dtype, scale=scale), _offsets(off)
    o, lse = op.forward(q.cuda(), k.cuda(), v.cuda(), st)
    dq, dk, dv = op.backward(q.cuda(), k.cuda(), v.cuda(), st, do.cuda())
    Q, K, V, G = (_np(t) for t in (q, k, v, do))
    r, got = HALF[dtype], dict(o=_np(o), lse=_np(lse), dq=_np(dq), dk=_np(dk), dv=_np(dv))
    want_dv, tol_dv, tol_dk = np.zeros((T, d)), np.zeros((T, d)), np.zeros((T, d))
    for b, e in zip(off, off[1:]):
        for h in range(H):
            S = scale * (Q[b:e, h] @ K[b:e, 0].T)
            S = np.where(np.tril(np.ones((e - b, e - b), bool)), S, -np.inf)
            at = S.argmax(1)
            top = np.sort(S, 1)[:, -2:]
            if e - b > 1:                  # (the input is what it is meant to be: gaps beyond any rounding of S)
                assert (top[1:, 1] - top[1:, 0] > 200 + 2.0 ** -11 * top[1:, 1]).all()
            at_key = b + at
            assert np.array_equal(got["o"][b:e, h], V[at_key, 0]), (order, log2_score, "o")
            m = top[:, -1]
            size_s = scale * (np.abs(Q[b:e, h]) * np.abs(K[at_key, 0])).sum(1)
            assert (np.abs(got["lse"][h, b:e] - m) <= (d + 8) * U * size_s + 8 * U * np.abs(m)).all()
            e_dS = 2 * (d + 8) * U * (np.abs(G[b:e, h]) * np.abs(V[at_key, 0])).sum(1) * (1 + 2 * r)
            assert (np.abs(got["dq"][b:e, h]) <= (scale * e_dS)[:, None] * np.abs(K[at_key, 0]) * (1 + 2 * r)).all()
            np.add.at(want_dv, at_key, G[b:e, h])
            np.add.at(tol_dv, at_key, np.abs(G[b:e, h]))
            np.add.at(tol_dk, at_key, (scale * e_dS)[:, None] * np.abs(Q[b:e, h]))
        assert not got["dq"][b].any()                                             # a first row's only key
    assert (np.abs(got["dv"][:, 0] - want_dv) <= (r + 2 * T * U) * tol_dv + r * np.abs(want_dv)).all()
    assert (np.abs(got["dk"][:, 0]) <= tol_dk * (1 + 2 * r + 2 * T * U)).all()


@pytest.mark.parametrize("dtype,d", [(BF, 64), (BF, 128), (BF, 33), (F32, 128)])
def test_first_rows_of_equal_queries_and_keys(dtype, d):
    """q = k of magnitude 3e4 and more: each row's own score is the largest; sequences of one token and of several."""
    import paper_2510_04206_amd as P
    T, off = 400, [*range(0, 65), 100, 101, 230, 400]
    for size in (3e4, 1e12):
        log(f"attention q = k of {size} {dtype} {d}")
        g = torch.Generator().manual_seed(d)
        x = (size * torch.randn(T, 1, d, generator=g)).to(dtype)
        v, do = torch.randn(T, 1, d, generator=g).to(dtype), torch.randn(T, 1, d, generator=g).to(dtype)
        op, st = P.PackedAttention(T, 1, 1, d, dtype), _offsets(off)
        o, _ = op.forward(x.cuda(), x.cuda(), v.cuda(), st)
        dq, dk, dv = op.backward(x.cuda(), x.cuda(), v.cuda(), st, do.cuda())
        S, at = _np(x)[:, 0] @ _np(x)[:, 0].T * d ** -0.5, np.arange(T)
        for b, e in zip(off, off[1:]):
            at[b:e] = b + np.where(np.tril(np.ones((e - b, e - b), bool)), S[b:e, b:e], -np.inf).argmax(1)
        first = np.array(off[:-1])
        assert np.array_equal(_np(o)[first], _np(v)[first]) and not dq[first].any()
        assert np.array_equal(_np(o), _np(v)[at])
        assert all(bool(torch.isfinite(t.float()).all()) for t in (dq, dk, dv))
        ones = np.array([b for b, e in zip(off, off[1:]) if e == b + 1])
        assert np.array_equal(_np(dv)[ones], _np(do)[ones])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 80, 128])
def test_other_rows_keep_their_bits(dtype, d):
    """A sequence of huge scores in the same tiles: the others' results have the bits that they have without."""
    import paper_2510_04206_amd as P
    from test_gpu_attention import _make
    T, off = 360, [0, 100, 180, 360]
    log(f"attention huge scores beside others {dtype} {d}")
    q, k, v, do = (t.cuda() for t in _make(T, 4, 2, d, dtype))
    op, st = P.PackedAttention(T, 4, 2, d, dtype), _offsets(off)
    run = lambda: [t.clone() for t in (*op.forward(q, k, v, st), *op.backward(q, k, v, st, do))]   # noqa: E731
    want = run()
    k[100:180] *= 2.0 ** 40
    got = run()
    keep = [*range(100), *range(180, T)]
    for i, (a, b) in enumerate(zip(got, want)):
        assert torch.equal(a[:, keep] if i == 1 else a[keep], b[:, keep] if i == 1 else b[keep]), i
        assert torch.isfinite(a.float()).all()
