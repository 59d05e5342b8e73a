"""Newton-Schulz products through every launch they can take, against the formula in 64 bits.

Bounds as in test_gpu_newton_schulz.py (matrices of noise): 4e-3 of the result's norm for bf16, 3 times
torch's fp32 error and 1e-6 for fp32.  A tile that is missing or in another's place is off by about its
entries' size: every block of 64 x 64 is held to a tenth of the root mean square of all entries.
"""
import math

import pytest
import torch

import ns_launches
from helpers import log

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
A, B, C = 3.4445, -4.7750, 2.0315


def _ns(x):
    if x.shape[0] > x.shape[1]:
        return _ns(x.t().contiguous()).t().contiguous()
    x = x / (x.double().square().sum().sqrt() + 1e-7).to(x.dtype)
    for _ in range(5):
        g = x @ x.t().contiguous()
        x = A * x + (B * g + C * (g @ g)) @ x
    return x


def _blocks(t):
    """Norms of the blocks of 64 x 64 (a border's may be smaller)."""
    m, n = t.shape
    t = torch.nn.functional.pad(t.square(), (0, -n % 64, 0, -m % 64))
    return t.view(t.shape[0] // 64, 64, t.shape[1] // 64, 64).sum((1, 3)).sqrt()


def _near(got, want, tol, what):
    off = got.double() - want
    e = float(off.norm() / want.norm())
    assert math.isfinite(e) and e <= tol, (what, e, tol)
    size = _blocks(torch.full_like(want, float(want.norm()) / want.numel() ** 0.5))
    assert not bool((_blocks(off) > 0.1 * size).any()), what
    return e


def _noise(batch, m, n, seed):
    return torch.randn(batch, m, n, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


@pytest.mark.parametrize("batch,r,k,f32", ns_launches.SIZES)
@pytest.mark.parametrize("tall", [False, True])
def test_orthogonalize(batch, r, k, f32, tall):
    import paper_2510_04206_amd as P
    m, n = (k, r) if tall else (r, k)
    log(f"orthogonalize {batch} x {m} x {n} f32 {f32}")
    x = _noise(batch, m, n, r)
    op = P.Orthogonalize(m, n, out_dtype=F32 if f32 else BF, batch=batch)
    op.out.fill_(float("nan"))
    got = op(x)
    worst = 0.0
    for i in range(batch):
        want = _ns(x[i].double())
        tol = 4e-3
        if f32:
            tol = 3 * float((_ns(x[i]).double() - want).norm() / want.norm()) + 1e-6
        worst = max(worst, _near(got[i], want, tol, i) / tol)
    log(f"  {worst:.2f} of the bound")


@pytest.mark.parametrize("batch,r,k,f32", ns_launches.SIZES)
@pytest.mark.parametrize("tall", [False, True])
def test_muon(batch, r, k, f32, tall):
    """The weight's update behind every launch: rows of a wider buffer, which keeps its other values.
    Off by 2e-3 (fp32: 2e-5) of lr scale |O| and the result's rounding, 2^-8 (2^-24 twice) of itself."""
    import paper_2510_04206_amd as P
    m, n = (k, r) if tall else (r, k)
    log(f"muon {batch} x {m} x {n} f32 {f32}")
    dtype = F32 if f32 else BF
    grad, mom = _noise(batch, m, n, k), _noise(batch, m, n, k + 1)
    wide = torch.full((batch, m, n + 3), 7.0, dtype=dtype, device="cuda")
    w = wide[..., :n]
    w.copy_(_noise(batch, m, n, k + 2) / k ** 0.5)
    old, was = w.clone(), mom.clone()
    op = P.MuonStep(m, n, param_dtype=dtype, batch=batch, momentum=0.9, weight_decay=0.5, scale=1.5)
    op(w, grad, mom, 0.5)
    assert bool((wide[..., n:] == 7.0).all())
    worst = 0.0
    for i in range(batch):
        m64 = 0.9 * was[i].double() + grad[i].double()
        assert float(((mom[i].double() - m64).abs() - 2.0 ** -22 * (m64.abs() + was[i].double().abs())).max()) <= 0
        o = _ns(grad[i].double() + 0.9 * m64)
        want = (1 - 0.5 * 0.5) * old[i].double() - 0.5 * 1.5 * o
        tol = ((2e-5 if f32 else 2e-3) * 0.5 * 1.5 * float(o.norm() / want.norm()) +
               (2.0 ** -23 if f32 else 2.0 ** -8))
        worst = max(worst, _near(w[i], want, tol, i) / tol)
    log(f"  {worst:.2f} of the bound")
