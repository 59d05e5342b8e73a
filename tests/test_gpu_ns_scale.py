"""Newton-Schulz products of matrices whose norm lies near the ends of fp32's range.

Bounds: a zero matrix gives 0 whatever eps is; otherwise, relative in the Frobenius norm, 4e-3 for a
bf16 result and for an fp32 one 3 times what torch fp32 is off by on the same matrix scaled to
ordinary size, and 1e-6 (scaling by a power of two changes no rounding but those of subnormal inputs,
which both sides are given).
"""
import pytest
import torch

from helpers import log

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
A, B, C = 3.4445, -4.7750, 2.0315
# one workgroup; launches in two parts; (bf16) in one part, wide and tall
SIZES = [(40, 90), (128, 300), (130, 200), (333, 150)]


def _ns(x, eps):
    if x.shape[0] > x.shape[1]:
        return _ns(x.t().contiguous(), eps).t()
    x = x / (x.double().square().sum().sqrt() + eps).to(x.dtype)
    for _ in range(5):
        g = x @ x.t().contiguous()
        x = A * x + (B * g + C * (g @ g)) @ x
    return x


def _rel(got, want):
    return float((got.double().cpu() - want).norm() / want.norm())


@pytest.mark.parametrize("m,n", SIZES)
@pytest.mark.parametrize("out", [BF, F32])
@pytest.mark.parametrize("eps", [1e-7, 1e-36, 1e-45])
def test_zero_matrix_gives_zero(m, n, out, eps):
    import paper_2510_04206_amd as P
    log(f"orthogonalize zeros {m} x {n} -> {out}, eps {eps}")
    x = torch.zeros(3, m, n, device="cuda")
    x[1] = torch.randn(m, n, generator=torch.Generator().manual_seed(m)).cuda()
    op = P.Orthogonalize(m, n, out_dtype=out, batch=3, eps=eps)
    op.out.fill_(float("nan"))
    got = op(x)
    assert not got[0].any() and not got[2].any()
    assert torch.equal(got[1], P.Orthogonalize(m, n, out_dtype=out, eps=eps)(x[1]))


@pytest.mark.parametrize("m,n", SIZES)
@pytest.mark.parametrize("out", [BF, F32])
def test_zero_gradient_only_decays_the_weight(m, n, out):
    """No gradient and no momentum: W <- (1 - lr wd) W, rounded once."""
    import paper_2510_04206_amd as P
    log(f"muon of zeros {m} x {n} {out}")
    w = torch.randn(m, n, generator=torch.Generator().manual_seed(n)).to(out).cuda()
    z = torch.zeros(m, n, device="cuda")
    want = (w.float() * (1 - 0.5 * 0.25)).to(out)
    P.MuonStep(m, n, param_dtype=out, weight_decay=0.25, eps=1e-40)(w, z, z.clone(), 0.5)
    assert torch.equal(w, want)


@pytest.mark.parametrize("m,n", SIZES)
@pytest.mark.parametrize("out", [BF, F32])
@pytest.mark.parametrize("log2", [-140, -126, -60, 60, 124])
def test_any_scale(m, n, out, log2):
    """Entries of 2^log2, down to subnormal ones, with an eps that does not count."""
    import paper_2510_04206_amd as P
    log(f"orthogonalize {m} x {n} -> {out}, entries of 2^{log2}")
    x = (torch.randn(m, n, generator=torch.Generator().manual_seed(7 * m + n)).double() * 2.0 ** log2).float()
    want = _ns(x.double(), 2.0 ** -149)
    unit = (x.double() * 2.0 ** -log2).float()            # exact
    tol = 4e-3 if out == BF else 3 * _rel(_ns(unit, 0.0), want) + 1e-6
    e = _rel(P.Orthogonalize(m, n, out_dtype=out, eps=1e-45)(x.cuda()), want)
    log(f"  off by {e:.2e} (bound {tol:.2e})")
    assert e <= tol
