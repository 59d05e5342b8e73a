"""Newton-Schulz orthogonalisation and the optimiser step against their formulas in 64 bits.

Bounds, relative in the Frobenius norm:
  bf16 result  4e-3: the products' operands in 11 bits leave at most 2e-3 (documented; the spread
               of inputs below has 1.6e-3 in a simulation of the roundings), the result's own
               rounding 2^-9;
  fp32 result  "as exact as fp32 products": 3 times what the same formula in torch fp32 on the CPU
               is off by on the same input, and 1e-6.
"""
import math

import pytest
import torch

from helpers import log

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
QUINTIC = (3.4445, -4.7750, 2.0315)
BF, F32 = torch.bfloat16, torch.float32


def _ns(x, steps=5, coeffs=QUINTIC, eps=1e-7):
    """The formula in x's own precision, on the side with fewer rows."""
    a, b, c = coeffs
    if x.shape[0] > x.shape[1]:
        return _ns(x.t().contiguous(), steps, coeffs, eps).t()
    x = x / ((x.double().square().sum().sqrt() + eps).to(x.dtype))
    for _ in range(steps):
        g = x @ x.t().contiguous()
        x = a * x + (b * g + c * (g @ g)) @ x
    return x


def _rel(got, want):
    want = want.double().cpu()
    return float((got.double().cpu() - want).norm() / max(float(want.norm()), 1e-300))


def _matrix(m, n, kind, seed=0):
    g = torch.Generator().manual_seed(seed + 7919 * m + n)
    x = torch.randn(m, n, generator=g)
    k = min(m, n)
    if kind == "flat":
        return x
    s = {"steep": 1.0 / torch.arange(1, k + 1).float() ** 2,
         "few": torch.where(torch.arange(k) < 8, 1.0, 1e-3)}[kind]
    u = torch.linalg.qr(torch.randn(m, k, generator=g))[0]
    v = torch.linalg.qr(torch.randn(n, k, generator=g))[0]
    return (u * s) @ v.t()


def _check(out, x, tol32, **kw):
    want = _ns(x.double().cuda(), **kw)
    e = _rel(out, want)
    if out.dtype == BF:
        bound = 4e-3
    else:
        bound = 3 * tol32 + 1e-6
    log(f"  off by {e:.2e} (bound {bound:.2e})")
    assert math.isfinite(e) and e <= bound
    return e


def _off32(x, **kw):
    return _rel(_ns(x.float().cpu(), **kw), _ns(x.double().cuda(), **kw))


SIZES = [(1, 1), (1, 7), (9, 1), (16, 16), (33, 65), (64, 64), (65, 129), (130, 64), (128, 512),
         (100, 1000), (255, 257), (1001, 400), (512, 512), (64, 4097)]


@pytest.mark.parametrize("m,n", SIZES)
@pytest.mark.parametrize("out", [BF, F32])
@pytest.mark.parametrize("kind", ["flat", "steep", "few"])
def test_sizes(m, n, out, kind):
    import paper_2510_04206_amd as P
    log(f"orthogonalize {m} x {n} {kind} -> {out}")
    x = _matrix(m, n, kind)
    op = P.Orthogonalize(m, n, out_dtype=out)
    op.out.fill_(float("nan"))
    _check(op(x.cuda()), x, _off32(x) if out == F32 else 0.0)
    if out == BF:
        _check(op(x.bfloat16().cuda()), x.bfloat16().float(), 0.0)


# a stack of middle size and single matrices whose products take the larger tiles
@pytest.mark.parametrize("m,n,batch", [(1100, 1501, 1), (700, 900, 4), (260, 2050, 9), (3700, 3590, 1)])
@pytest.mark.parametrize("out", [BF, F32])
def test_larger_tiles(m, n, batch, out):
    import paper_2510_04206_amd as P
    log(f"orthogonalize {batch} x {m} x {n} -> {out}")
    x = torch.stack([_matrix(m, n, "flat", seed=i) for i in range(batch)])
    got = P.Orthogonalize(m, n, out_dtype=out, batch=batch)(x.cuda())
    for i in {0, batch - 1}:
        _check(got[i], x[i], _off32(x[i]) if out == F32 else 0.0)


# both sides of the sizes that one workgroup holds (64 rows, 256 columns), several to a stack
@pytest.mark.parametrize("m,n", [(64, 256), (256, 64), (64, 257), (63, 129), (65, 256), (2, 200),
                                 (255, 40)])
@pytest.mark.parametrize("out", [BF, F32])
def test_small_stacks(m, n, out):
    import paper_2510_04206_amd as P
    log(f"orthogonalize 5 x {m} x {n} -> {out}")
    x = torch.stack([_matrix(m, n, kind, seed=i) for i, kind in
                     enumerate(("flat", "steep", "few", "flat", "steep"))])
    got = P.Orthogonalize(m, n, out_dtype=out, batch=5)(x.cuda())
    for i in range(5):
        _check(got[i], x[i], _off32(x[i]) if out == F32 else 0.0)


@pytest.mark.parametrize("out", [BF, F32])
def test_transposed_input_transposes_the_result(out):
    import paper_2510_04206_amd as P
    log("orthogonalize of a transpose")
    x = _matrix(200, 333, "flat").cuda()
    a = P.Orthogonalize(200, 333, out_dtype=out)(x)
    b = P.Orthogonalize(333, 200, out_dtype=out)(x.t().contiguous())
    assert torch.equal(a, b.t())


def test_strides_and_starts():
    import paper_2510_04206_amd as P
    from paper_2510_04206_amd import _binding as B
    log("orthogonalize strides")
    b, m, n = 3, 70, 45
    x = torch.stack([_matrix(m, n, "flat", seed=i) for i in range(b)]).cuda()
    op = P.Orthogonalize(m, n, out_dtype=F32, batch=b)
    want = op(x).clone()
    wide = torch.full((b, m + 3, n + 5), float("nan"), device="cuda")
    view = wide[:, 1:m + 1, 3:n + 3]
    view.copy_(x)
    assert torch.equal(op(view), want)
    # the same matrix for every member of the stack
    assert torch.equal(op(x[1].expand(b, m, n))[2], want[1])
    # rows of the result further apart, from an odd element on
    out = torch.full((b * m * (n + 2) + 1,), 7.0, device="cuda")
    o = out[1:].view(b, m, n + 2)
    B.agrl_orthogonalize(b, m, n, 1, x, n, m * n, 1, op.ns, op.workspace, op.ws_bytes, o[:, :, :n],
                         n + 2, m * (n + 2))
    assert torch.equal(o[:, :, :n], want) and bool((o[:, :, n:] == 7.0).all()) and float(out[0]) == 7.0


def test_a_vector_and_other_polynomials():
    """One row: p applied `steps` times to 1, in the row's direction; and the cubic that converges."""
    import paper_2510_04206_amd as P
    log("orthogonalize vector, cubic")
    x = _matrix(1, 300, "flat")
    s = 1.0
    for _ in range(5):
        s = QUINTIC[0] * s + QUINTIC[1] * s ** 3 + QUINTIC[2] * s ** 5
    got = P.Orthogonalize(1, 300, out_dtype=F32)(x.cuda())
    assert _rel(got, s * x.double() / x.double().norm()) <= 2e-6
    x = _matrix(48, 96, "flat")
    kw = dict(steps=12, coeffs=(1.5, -0.5, 0.0))
    got = P.Orthogonalize(48, 96, out_dtype=F32, **kw)(x.cuda())
    _check(got, x, _off32(x, **kw), **kw)
    got = got.double()
    assert float((got @ got.t().contiguous() - torch.eye(48, device="cuda").double()).abs().max()) <= 2e-5
    _check(P.Orthogonalize(48, 96, out_dtype=BF, steps=1)(x.cuda()), x, 0.0, steps=1)


def test_scales_zero_and_non_finite():
    import paper_2510_04206_amd as P
    log("orthogonalize scales, zeros, non-finite")
    x = torch.stack([_matrix(40, 90, "flat", seed=i) for i in range(4)])
    op = P.Orthogonalize(40, 90, out_dtype=F32, batch=4)
    base = op(x.cuda()).clone()
    # sums of squares past fp32's range; a norm of 0.015, where eps counts 7e-6 (by the formula)
    for s in (2.0 ** 80, 2.0 ** -12):
        want = torch.stack([_ns((t * s).double()) for t in x])
        assert _rel(op((x * s).cuda()), want) <= 1e-5
    # entries of 1e-30 without an eps of consequence
    tiny = P.Orthogonalize(40, 90, out_dtype=F32, batch=4, eps=1e-37)
    assert _rel(tiny((x * 2.0 ** -100).cuda()), base) <= 1e-5
    bad = x.clone()
    bad[0] = 0.0
    bad[1, 3, 4] = float("nan")
    bad[2, 39, 89] = float("inf")
    got = op(bad.cuda())
    assert not got[0].any() and torch.isnan(got[1]).all() and torch.isnan(got[2]).all()
    assert torch.equal(got[3], base[3])


@pytest.mark.parametrize("grad_dtype,param_dtype", [(F32, F32), (BF, F32), (F32, BF), (BF, BF)])
@pytest.mark.parametrize("m,n,batch,nesterov", [(70, 200, None, True), (300, 128, None, False),
                                                (96, 96, 3, True), (50, 333, 2, True),
                                                (201, 64, None, False), (1300, 1100, None, True)])
def test_muon_steps(grad_dtype, param_dtype, m, n, batch, nesterov):
    """Three steps.  Momentum: one rounding of each term a step, 4 u of their sizes.  Parameter:
    lr scale O off by the bounds above, and u (bf16: 2^-9) of itself a step."""
    import paper_2510_04206_amd as P
    log(f"muon {m} x {n} batch {batch} grad {grad_dtype} param {param_dtype} nesterov {nesterov}")
    lr, mu, wd = 0.05, 0.9, 0.2
    shape = (m, n) if batch is None else (batch, m, n)
    g = torch.Generator().manual_seed(m)
    w = (0.1 * torch.randn(shape, generator=g)).to(param_dtype)
    mom = torch.randn(shape, generator=g) * 1e-3
    wd64, mom64, size = w.double().cuda(), mom.double().cuda(), mom.double().abs().cuda()
    wide = torch.full((*shape[:-1], n + 3), 7.0, dtype=param_dtype, device="cuda")
    par, buf = wide[..., :n], mom.cuda()
    par.copy_(w)
    op = P.MuonStep(m, n, param_dtype=param_dtype, batch=batch, momentum=mu, nesterov=nesterov,
                    weight_decay=wd)
    scale = math.sqrt(max(1.0, m / n))
    bound = 0.0
    for k in range(3):
        grad = (torch.randn(shape, generator=g) * 1e-3).to(grad_dtype)
        assert op(par, grad.cuda(), buf, lr) is par
        g64 = grad.double().cuda()
        mom64 = mu * mom64 + g64
        size = mu * size + g64.abs()
        u = g64 + mu * mom64 if nesterov else mom64
        o = torch.stack([_ns(t) for t in u.view(-1, m, n)]).view(shape)
        wd64 = (1 - lr * wd) * wd64 - lr * scale * o
        off = 2e-3 if param_dtype == BF else 2e-5
        bound += (off * lr * scale * float(o.norm()) +
                  (2.0 ** -9 if param_dtype == BF else 2 * U) * float(wd64.norm()))
        assert float(((buf.double() - mom64).abs() - 4 * (k + 1) * U * size).max()) <= 0
        e = float((par.double() - wd64).norm())
        log(f"  step {k}: parameter off by {e / bound:.2f} of the bound")
        assert e <= bound
    assert bool((wide[..., n:] == 7.0).all())


def test_muon_scale_and_plain_sum():
    """scale given, no decay, mu 0: the parameter moves by lr scale O(grad)."""
    import paper_2510_04206_amd as P
    log("muon scale")
    x = _matrix(64, 32, "flat").cuda()
    o = P.Orthogonalize(64, 32, out_dtype=F32)(x)
    w, buf = torch.zeros(64, 32, device="cuda"), torch.full((64, 32), 5.0, device="cuda")
    P.MuonStep(64, 32, momentum=0.0, nesterov=False, scale=0.25)(w, x, buf, 0.5)
    assert torch.equal(buf, x) and _rel(w, -0.125 * o) <= 2 * U


def test_stream_repeat_and_graph():
    import paper_2510_04206_amd as P
    log("orthogonalize stream and graph")
    x = _matrix(300, 500, "flat").cuda()
    w0 = torch.randn(300, 500, device="cuda")
    op, mu = P.Orthogonalize(300, 500), P.MuonStep(300, 500)
    want = op(x).clone()
    torch.cuda.synchronize()
    assert torch.equal(op(x), want)
    s = torch.cuda.Stream()
    other = P.Orthogonalize(300, 500)
    got = other(x, stream=s)
    s.synchronize()
    assert torch.equal(got, want)
    w, buf = w0.clone(), torch.zeros(300, 500, device="cuda")
    we, bufe = w0.clone(), torch.zeros(300, 500, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        op(x)
        mu(w, x, buf, 0.1)
    for k in range(3):
        x.copy_(_matrix(300, 500, "flat", seed=k))
        op.out.fill_(3.0)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(op.out, other(x))
        mu(we, x, bufe, 0.1)
        torch.cuda.synchronize()
        assert torch.equal(w, we) and torch.equal(buf, bufe)


def test_api_refusals():
    import paper_2510_04206_amd as P
    log("orthogonalize refusals")
    op = P.Orthogonalize(8, 16)
    x = torch.zeros(8, 16, device="cuda")
    with pytest.raises(ValueError):
        op(x.t())
    with pytest.raises(ValueError):
        op(torch.zeros(8, 32, device="cuda")[:, ::2])
    with pytest.raises(TypeError):
        op(x.half())
    with pytest.raises(ValueError):
        op(x.cpu())
    with pytest.raises(TypeError):
        P.Orthogonalize(8, 16, out_dtype=torch.float16)
    with pytest.raises(ValueError):
        P.Orthogonalize(8, 16, steps=0)
    with pytest.raises(P.AgrlError):
        P.Orthogonalize(8, 16, coeffs=(float("nan"), 0.0, 0.0))(x)
    mu = P.MuonStep(8, 16)
    with pytest.raises(TypeError):
        mu(x.bfloat16(), x, x.clone(), 0.1)
    with pytest.raises(TypeError):
        mu(x, x, x.bfloat16(), 0.1)
    with pytest.raises(P.AgrlError):
        mu(x, x.clone(), x.clone(), float("inf"))
    with pytest.raises(ValueError):
        mu(x, x.clone(), torch.zeros(8, 32, device="cuda")[:, :16], 0.1)   # momentum is contiguous
