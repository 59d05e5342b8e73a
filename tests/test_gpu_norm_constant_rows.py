"""Layer norm of constant rows far from zero.

A constant row's variance is 0 up to the roundings of a mean (64 u |x|, u = 2^-24), squared, and never
below 0, so rstd lies in (0, 1 / sqrt(eps)] up to 64 u.
"""
import pytest
import torch

from helpers import log

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.mark.parametrize("d", [2, 97, 600, 1025, 1777, 3001, 4991, 8191, 16383])
@pytest.mark.parametrize("size", [1e3, 1e8, 1e12, 1e15])
def test_constant_rows_far_from_zero(d, size):
    import paper_2510_04206_amd as P
    log(f"norm constant rows of {size:g}, d={d}")
    T, eps = 400, 1e-5
    v = size * (0.5 + 1.5 * torch.rand(T, generator=torch.Generator().manual_seed(d)))
    x = v[:, None].expand(T, d).contiguous().cuda()
    y, mean, rstd = P.TokenNorm(T, d, torch.float32, eps=eps, grads=False).forward(x)
    assert bool(torch.isfinite(y).all()) and bool(torch.isfinite(rstd).all())
    v = v.double().cuda()
    assert bool(((mean.double() - v).abs() <= 64 * U * v).all())
    assert bool((rstd > 0).all()) and float(rstd.max()) <= (1 + 64 * U) / eps ** 0.5
    assert bool((y.double().abs() <= 64 * U * v[:, None] * rstd.double()[:, None] + 1e-30).all())
