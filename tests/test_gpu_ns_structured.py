"""Newton-Schulz products of matrices whose entries repeat, where roundings add up instead of averaging.

Blocks of ones on the diagonal, an outer product of signs, the identity: all entries of X, of A and of B
that belong to a singular value carry the same relative rounding errors, so a singular value s moves
by the scalar recursion with, a step, an error u at each of X, A and B on top of the slope p'(s) times
the error before.  bound() sums these to first order with the worst signs; 1.2 of it covers the second
order (the errors are below 7e-2).  u is
  bf16 result, more than 128 rows   2^-11, operands in 11 bits, and 2^-8 of the result's own rounding (all entries alike)
  otherwise                         2^-22 of an operand in two parts, 2^-22 of the product left out,
                                    2^-24 for each of k / 32 + 8 sums (and the result's own 2^-24 or 2^-8)
"""
import numpy as np
import pytest
import torch

from helpers import log

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
A, B, C = 3.4445, -4.7750, 2.0315


def bound(s, u, last_steps):
    """Worst error of the polynomial's five steps over the singular values s, relative in the norm.
    last_steps: the multiples of I that are added to B in the last two steps (0 in two parts)."""
    e = np.zeros_like(s)
    for k in range(5):
        sg = last_steps[k - 3] if k >= 3 else 0.0
        d_x = abs(3 * B * s ** 3 + 5 * C * s ** 5 + sg * s)
        d_a = abs(B * s ** 3 + 2 * C * s ** 5)
        d_b = abs(B * s ** 3 + C * s ** 5 + sg * s)
        # (the state itself, hi + lo, is rounded to 22 bits)
        e = abs(A + 3 * B * s ** 2 + 5 * C * s ** 4) * e + u * (d_x + d_a + d_b) + 2.0 ** -22 * abs(A * s)
        s = A * s + B * s ** 3 + C * s ** 5
    return 1.2 * np.linalg.norm(e) / np.linalg.norm(s)


def _matrix(m, n, kind):
    if kind == "eye":
        return torch.eye(m, n)
    if kind == "signs":
        g = torch.Generator().manual_seed(m + n)
        return torch.sign(torch.randn(m, 1, generator=g)) @ torch.sign(torch.randn(1, n, generator=g))
    x = torch.zeros(m, n)
    k = int(kind)
    for i in range(k):
        x[i * m // k:(i + 1) * m // k, i * n // k:(i + 1) * n // k] = 1.0
    return x


def _exact(x):
    if x.shape[0] > x.shape[1]:
        return _exact(x.t().contiguous()).t()
    x = x / (x.norm() + 1e-7)
    for _ in range(5):
        g = x @ x.t().contiguous()
        x = A * x + (B * g + C * (g @ g)) @ x
    return x


@pytest.mark.parametrize("m,n", [(40, 90), (128, 300), (129, 200), (300, 500), (1000, 257), (512, 512), (1000, 1000)])
@pytest.mark.parametrize("out", [BF, F32])
@pytest.mark.parametrize("kind", ["1", "2", "4", "12", "signs", "eye"])
def test_repeated_entries(m, n, out, kind):
    import paper_2510_04206_amd as P
    log(f"orthogonalize {kind} {m} x {n} -> {out}")
    x = _matrix(m, n, kind)
    want = _exact(x.double().cuda())
    s = torch.linalg.svdvals(x.double()).numpy()
    s = s[s > 1e-9 * s[0]] / np.linalg.norm(s)
    if out == BF and min(m, n) > 128:
        tol = bound(s, 2.0 ** -11, (-0.5 * (B + C), A)) + 2.0 ** -8
    else:
        k = max(m, n)
        tol = bound(s, 2.0 ** -21 + (k / 32 + 8) * 2.0 ** -24, (0.0, 0.0)) + (2.0 ** -8 if out == BF else 2.0 ** -24)
    got = P.Orthogonalize(m, n, out_dtype=out)(x.cuda())
    e = float((got.double() - want).norm() / want.norm())
    log(f"  off by {e:.2e} (bound {tol:.2e})")
    assert e <= tol
