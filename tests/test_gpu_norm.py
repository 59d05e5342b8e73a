"""Layer and RMS norm, forward and backward, against their definitions in 64 bits.

Bounds, with u = 2^-24 and the row's largest |x| times rstd written X.  A lane adds at most
24 terms in order, then 6 + 16 partial sums join: a mean is off by at most 46 u max|x|, a
variance (taken about the mean) by 48 u of itself, the quotients and products by a few u:
  rstd   64 u relative
  y      64 u (|w| (|xh| + X) + |b|), and for bf16 one rounding, 2^-8 |y| at most
  dx     128 u rstd (|g| + mean|g| + (|xh| + X) mean|g xh|), and the same rounding
  dw     (128 + rows in order) u sum |dy| (|xh| + X);  db likewise with sum |dy|
where a team adds its rows in order (at most T / 512 of them, rounded up) and 512 / 16 partial
sums follow.
"""
import numpy as np
import pytest
import torch

from helpers import log

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
EPS = 1e-5


def _ref(x, w, b, mask, dy, kind, eps=EPS):
    """Everything in 64 bits on the CPU, with the bounds above."""
    live = np.ones(x.shape[0], bool) if mask is None else mask.astype(bool)
    x, dy = np.where(live[:, None], x, 0.0), np.where(live[:, None], dy, 0.0)
    d = x.shape[1]
    mean = x.mean(1) if kind == "layer" else np.zeros(len(x))
    var = ((x - mean[:, None]) ** 2).mean(1)
    rstd = np.where(live, 1 / np.sqrt(var + eps), 0.0)
    xh = (x - mean[:, None]) * rstd[:, None]
    X = (np.abs(x).max(1) * rstd)[:, None]
    y = np.where(live[:, None], xh * w + b, 0.0)
    g = dy * w
    c1 = g.mean(1, keepdims=True) if kind == "layer" else 0.0
    c2 = (g * xh).mean(1, keepdims=True)
    dx = rstd[:, None] * (g - c1 - xh * c2)
    n = 128 + -(-x.shape[0] // 512) + 32
    return dict(
        y=y, mean=np.where(live, mean, 0.0), rstd=rstd, dx=dx, dw=(dy * xh).sum(0), db=dy.sum(0),
        t_y=64 * U * (np.abs(w) * (np.abs(xh) + X) + np.abs(b)),
        t_mean=64 * U * np.abs(x).max(1), t_rstd=64 * U * rstd,
        t_dx=128 * U * rstd[:, None] * (np.abs(g) + np.abs(g).mean(1, keepdims=True) +
                                        (np.abs(xh) + X) * np.abs(g * xh).mean(1, keepdims=True)),
        t_dw=n * U * (np.abs(dy) * (np.abs(xh) + X)).sum(0), t_db=n * U * np.abs(dy).sum(0),
        live=live, d=d)


def _np(t):
    return t.detach().double().cpu().numpy()


def _near(got, want, tol, dtype, what):
    tol = tol + 1e-30 + (2.0 ** -8 * np.abs(want) if dtype == torch.bfloat16 else 0.0)
    off = np.abs(_np(got) - want) / tol
    assert np.isfinite(_np(got)).all(), what
    assert off.max(initial=0.0) <= 1.0, (what, float(off.max()))
    return float(off.max(initial=0.0))


def _inputs(T, d, dtype, wdtype, dydtype, kind, mask, seed=0, shift=0.3, pitch=0):
    g = torch.Generator().manual_seed(seed + 1000 * T + d)
    mk = lambda *n: torch.randn(*n, generator=g)                                  # noqa: E731
    x = (mk(T, d) * torch.exp(mk(T, 1)) + shift).to(dtype)
    w, b = (1 + 0.3 * mk(d)).to(wdtype), (0.3 * mk(d)).to(wdtype)
    dy = (0.01 * mk(T, d)).to(dydtype)
    m = {"none": None, "some": (torch.rand(T, generator=g) < 0.4).to(torch.uint8),
         "dead": torch.zeros(T, dtype=torch.uint8)}[mask]
    dev = []
    for t in (x, dy):
        wide = torch.full((T, d + pitch), float("nan"), dtype=t.dtype, device="cuda")
        wide[:, :d] = t.cuda()
        dev.append(wide[:, :d])
    return x, w, b, m, dy, dev[0], dev[1]


def _run(T, d, dtype=torch.bfloat16, wdtype=torch.float32, dydtype=torch.float32, kind="layer",
         mask="none", affine=True, **kw):
    import paper_2510_04206_amd as P
    log(f"norm T={T} d={d} {dtype} w {wdtype} dy {dydtype} {kind} mask {mask} affine {affine} {kw}")
    x, w, b, m, dy, xd, dyd = _inputs(T, d, dtype, wdtype, dydtype, kind, mask, **kw)
    op = P.TokenNorm(T, d, dtype, kind=kind, eps=EPS, bias_grad=True)
    for t in (op.y, op.rstd, op.dx, op.dweight, op.dbias, op.mean):
        if t is not None:
            t.fill_(float("nan"))
    md = None if m is None else m.cuda()
    wd, bd = (w.cuda(), b.cuda()) if affine else (None, None)
    y, mean, rstd = op.forward(xd, wd, bd, md)
    dx, dw, db = op.backward(xd, wd, dyd, md)
    torch.cuda.synchronize()
    r = _ref(_np(x), _np(w) if affine else np.ones(d), _np(b) if affine else np.zeros(d),
             None if m is None else m.numpy(), _np(dy), kind)
    offs = [_near(y, r["y"], r["t_y"], dtype, "y"), _near(rstd, r["rstd"], r["t_rstd"], None, "rstd"),
            _near(dx, r["dx"], r["t_dx"], dtype, "dx"), _near(dw, r["dw"], r["t_dw"], None, "dw"),
            _near(db, r["db"], r["t_db"], None, "db")]
    if kind == "layer":
        offs.append(_near(mean, r["mean"], r["t_mean"], None, "mean"))
    log("  shares of the bounds: " + " ".join(f"{o:.2f}" for o in offs))
    dead = ~r["live"]
    for t in (y, dx):
        z = _np(t)[dead]
        assert not z.any() and not np.signbit(z).any()
    return op


# every team shape's first, last and odd lengths; one row, a few, more than a group of 64 per team
SHAPES = [(1, 1), (3, 7), (5, 8), (1, 257), (66, 512), (65, 513), (33, 1024), (7, 1025), (130, 2048),
          (9, 2049), (40, 4096), (3, 4097), (11, 6144), (5, 6145), (6, 8192), (3, 8193), (2, 16384),
          (1519, 256), (2100, 1001), (40000, 72)]


@pytest.mark.parametrize("T,d", SHAPES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_shapes(T, d, dtype, kind):
    _run(T, d, dtype, kind=kind)


@pytest.mark.parametrize("mask", ["some", "dead"])
@pytest.mark.parametrize("T,d", [(1, 65), (70, 300), (700, 2048), (2500, 5120), (70000, 40)])
def test_masks(T, d, mask):
    _run(T, d, mask=mask)


@pytest.mark.parametrize("dtype,wdtype,dydtype", [
    (torch.bfloat16, torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.bfloat16, torch.float32),
    (torch.float32, torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32, torch.bfloat16)])
@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_types(dtype, wdtype, dydtype, kind):
    _run(301, 1100, dtype, wdtype, dydtype, kind, "some")
    _run(301, 1100, dtype, wdtype, dydtype, kind, "some", affine=False)


@pytest.mark.parametrize("pitch", [1, 3, 64])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_strides(dtype, pitch):
    _run(77, 999, dtype, mask="some", pitch=pitch)
    _run(77, 1024, dtype, pitch=pitch)


@pytest.mark.parametrize("start", [1, 2, 3, 5])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_arrays_start_anywhere(dtype, start):
    """Inputs, outputs and parameters cut out of buffers at an odd element."""
    from paper_2510_04206_amd import _binding as B
    T, d = 50, 777
    log(f"norm start {start} {dtype}")
    x, w, b, _, dy, _, _ = _inputs(T, d, dtype, dtype, dtype, "layer", "none")
    code = B.dtype_code(x)
    cut = lambda t: torch.cat([t.new_zeros(start), t.reshape(-1)]).cuda()[start:]  # noqa: E731
    xd, wd, bd, dyd = cut(x), cut(w), cut(b), cut(dy)
    mean, rstd, dw, db = (cut(torch.full((n,), float("nan"))) for n in (T, T, d, d))
    y, dx = (cut(torch.full((T, d), float("nan"), dtype=dtype)) for _ in range(2))
    B.agrl_token_norm_fwd(T, d, 0, code, code, xd, d, wd, bd, None, EPS, y, d, mean, rstd)
    n = B.agrl_token_norm_bwd_workspace_size(T, d)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    B.agrl_token_norm_bwd(T, d, 0, code, code, code, xd, d, wd, None, dyd, d, mean, rstd, 0, ws, n,
                          dx, d, dw, db)
    r = _ref(_np(x), _np(w), _np(b), None, _np(dy), "layer")
    _near(y.view(T, d), r["y"], r["t_y"], dtype, "y")
    _near(dx.view(T, d), r["dx"], r["t_dx"], dtype, "dx")
    _near(dw, r["dw"], r["t_dw"], None, "dw")
    _near(db, r["db"], r["t_db"], None, "db")


@pytest.mark.parametrize("d", [200, 3000])
def test_row_far_from_zero(d):
    """A mean of 3e4 times the spread: a variance from sums of squares would lose it all."""
    _run(40, d, torch.float32, shift=3e4)


def test_rows_beyond_32_bit_offsets():
    from paper_2510_04206_amd import _binding as B
    d, ld, T = 130, (1 << 30) + 13, 5          # row 4 starts past 2^32 elements
    log("norm row stride 2^30 + 13")
    big = torch.empty(ld * (T - 1) + d, dtype=torch.bfloat16, device="cuda")
    xd = big.as_strided((T, d), (ld, 1))
    x, w, b, _, dy, _, dyd = _inputs(T, d, torch.bfloat16, torch.float32, torch.float32, "layer", "none")
    xd.copy_(x)
    mean, rstd = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    B.agrl_token_norm_fwd(T, d, 0, 0, 1, xd, ld, w.cuda(), b.cuda(), None, EPS, xd, ld, mean, rstd)
    r = _ref(_np(x), _np(w), _np(b), None, _np(dy), "layer")
    _near(xd, r["y"], r["t_y"], torch.bfloat16, "y over x")


def test_nan_and_inf_stay_where_they_are():
    """Masked rows are never read; a bad live row spoils its own outputs and the columns' sums."""
    import paper_2510_04206_amd as P
    T, d = 130, 640
    log("norm non-finite rows")
    x, w, b, _, dy, xd, dyd = _inputs(T, d, torch.bfloat16, torch.float32, torch.float32, "layer", "none")
    m = torch.ones(T, dtype=torch.uint8)
    m[::3] = 0
    op = P.TokenNorm(T, d, torch.bfloat16, eps=EPS)
    want = [t.clone() for t in op.forward(xd, w.cuda(), b.cuda(), m.cuda()) +
            op.backward(xd, w.cuda(), dyd, m.cuda())]
    xd[::3], dyd[::3] = float("nan"), float("inf")
    got = op.forward(xd, w.cuda(), b.cuda(), m.cuda()) + op.backward(xd, w.cuda(), dyd, m.cuda())
    for a, c in zip(got, want):
        assert torch.equal(a, c)
    xd[7, 5], xd[8, 6] = float("nan"), float("inf")
    y, mean, rstd, dx = (t.clone() for t in (*op.forward(xd, w.cuda(), b.cuda(), m.cuda()),
                                             op.backward(xd, w.cuda(), dyd, m.cuda())[0]))
    keep = torch.ones(T, dtype=torch.bool, device="cuda")
    keep[[7, 8]] = False
    for t, c in ((y, want[0]), (dx, want[3])):
        assert torch.equal(t[keep], c[keep])
        assert torch.isnan(t[7]).all() and torch.isnan(t[8]).any()


def test_constant_rows():
    import paper_2510_04206_amd as P
    log("norm constant rows")
    x = torch.arange(6.0).repeat_interleave(100).view(6, 100).cuda()
    w, b = torch.randn(100).cuda(), torch.randn(100).cuda()
    op = P.TokenNorm(6, 100, torch.float32, eps=EPS)
    y, mean, rstd = op.forward(x, w, b)
    # 64 u |x| of the mean, times rstd = 1 / sqrt(eps)
    assert float((y - b).abs().max()) <= 64 * U * 5 / EPS ** 0.5 * float(w.abs().max())
    assert float((rstd - EPS ** -0.5).abs().max()) <= 64 * U * EPS ** -0.5


def test_accumulate_empty_and_repeat():
    import paper_2510_04206_amd as P
    from paper_2510_04206_amd import _binding as B
    T, d = 3000, 321
    log("norm accumulate")
    x, w, b, m, dy, xd, dyd = _inputs(T, d, torch.bfloat16, torch.float32, torch.float32, "layer", "some")
    op = P.TokenNorm(T, d, torch.bfloat16, eps=EPS)
    op.forward(xd, w.cuda(), b.cuda(), m.cuda())
    dx, dw, db = (t.clone() for t in op.backward(xd, w.cuda(), dyd, m.cuda()))
    op.dweight.fill_(2.0), op.dbias.fill_(-1.0)
    got = op.backward(xd, w.cuda(), dyd, m.cuda(), accumulate=True)
    assert torch.equal(got[0], dx) and torch.equal(got[1], 2.0 + dw) and torch.equal(got[2], -1.0 + db)
    # no rows: sums of nothing, or what was there; no gradient asked for: no workspace
    z, k = torch.full((d,), 3.0, device="cuda"), torch.full((d,), 3.0, device="cuda")
    B.agrl_token_norm_bwd(0, d, 0, 0, 1, 1, None, d, None, None, None, d, None, None, 0, None, 0, None,
                          d, z, None)
    B.agrl_token_norm_bwd(0, d, 0, 0, 1, 1, None, d, None, None, None, d, None, None, 1, None, 0, None,
                          d, k, None)
    op.dx.fill_(7.0)
    B.agrl_token_norm_bwd(T, d, 0, 0, 1, 1, xd, d, w.cuda(), m.cuda(), dyd, d, op.mean, op.rstd, 0,
                          None, 0, op.dx, d, None, None)
    assert not z.any() and bool((k == 3.0).all()) and torch.equal(op.dx, dx)


def test_in_place():
    import paper_2510_04206_amd as P
    from paper_2510_04206_amd import _binding as B
    T, d = 300, 1200
    log("norm in place")
    x, w, b, m, dy, xd, dyd = _inputs(T, d, torch.float32, torch.float32, torch.float32, "rms", "some")
    op = P.TokenNorm(T, d, torch.float32, kind="rms", eps=EPS)
    y = op.forward(xd, w.cuda(), None, m.cuda())[0].clone()
    dx = op.backward(xd, w.cuda(), dyd, m.cuda())[0].clone()
    a, c = xd.clone(), dyd.clone()
    B.agrl_token_norm_fwd(T, d, 1, 1, 1, a, d, w.cuda(), None, m.cuda(), EPS, a, d, None, None)
    B.agrl_token_norm_bwd(T, d, 1, 1, 1, 1, xd, d, w.cuda(), m.cuda(), c, d, None, op.rstd, 0, None,
                          0, c, d, None, None)
    assert torch.equal(a, y) and torch.equal(c, dx)


@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_gradient_against_differences(kind):
    """Central differences of the 64-bit definition in random directions: 1e-4 of the size of the
    sum (h = 1e-5: truncation 1e-10, the fp32 gradient 1e-5 at most)."""
    import paper_2510_04206_amd as P
    T, d, h = 20, 90, 1e-5
    log(f"norm differences {kind}")
    x, w, b, m, dy, xd, dyd = _inputs(T, d, torch.float32, torch.float32, torch.float32, kind, "some")
    op = P.TokenNorm(T, d, torch.float32, kind=kind, eps=EPS, bias_grad=True)
    op.forward(xd, w.cuda(), b.cuda(), m.cuda())
    dx, dw, db = (_np(t) for t in op.backward(xd, w.cuda(), dyd, m.cuda()))
    v, X, Wt, Bs = _np(dy), _np(x), _np(w), _np(b)
    f = lambda X, Wt, Bs: (_ref(X, Wt, Bs, m.numpy(), v, kind)["y"] * v).sum()     # noqa: E731
    rng = np.random.default_rng(3)
    for _ in range(4):
        e, ew, eb = rng.standard_normal((T, d)), rng.standard_normal(d), rng.standard_normal(d)
        for grad, dirs in ((dx, (e, 0, 0)), (dw, (0, ew, 0)), (db, (0, 0, eb))):
            num = (f(X + h * dirs[0], Wt + h * dirs[1], Bs + h * dirs[2]) -
                   f(X - h * dirs[0], Wt - h * dirs[1], Bs - h * dirs[2])) / (2 * h)
            way = [q for q in dirs if not np.isscalar(q)][0]
            assert abs(num - (grad * way).sum()) <= 1e-4 * np.linalg.norm(grad) * np.linalg.norm(way) ** 0.5


def test_other_stream_and_graph():
    """A handle made on one stream and used on another, and replays of a captured pair of calls."""
    import paper_2510_04206_amd as P
    T, d = 2000, 1500
    log("norm stream and graph")
    x, w, b, m, dy, xd, dyd = _inputs(T, d, torch.bfloat16, torch.float32, torch.float32, "layer", "some")
    wd, bd, md = w.cuda(), b.cuda(), m.cuda()
    op = P.TokenNorm(T, d, torch.bfloat16, eps=EPS)
    want = [t.clone() for t in op.forward(xd, wd, bd, md) + op.backward(xd, wd, dyd, md)]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    other = P.TokenNorm(T, d, torch.bfloat16, eps=EPS)
    got = other.forward(xd, wd, bd, md, stream=s) + other.backward(xd, wd, dyd, md, stream=s)
    s.synchronize()
    for a, c in zip(got, want):
        assert torch.equal(a, c)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = op.forward(xd, wd, bd, md) + op.backward(xd, wd, dyd, md)
    for k in range(3):
        xd.mul_(2.0 if k else 1.0)
        for t in got:
            t.fill_(5.0)
        g.replay()
        torch.cuda.synchronize()
        eager = other.forward(xd, wd, bd, md) + other.backward(xd, wd, dyd, md)
        torch.cuda.synchronize()
        for a, c in zip(got, eager):
            assert torch.equal(a, c)


def test_api_refusals():
    import paper_2510_04206_amd as P
    log("norm refusals")
    op = P.TokenNorm(4, 32, torch.bfloat16, grads=False)
    x = torch.zeros(4, 32, dtype=torch.bfloat16, device="cuda")
    w = torch.ones(32, device="cuda")
    with pytest.raises(ValueError):
        op.forward(x[:3], w)
    with pytest.raises(TypeError):
        op.forward(x.float(), w)
    with pytest.raises(ValueError):
        op.forward(x, w[:31])
    with pytest.raises(TypeError):
        op.forward(x, w, w.bfloat16())                   # one type for weight and bias
    with pytest.raises(TypeError):
        op.forward(x, w, None, torch.ones(4, device="cuda"))
    with pytest.raises(ValueError):
        op.forward(torch.zeros(32, 4, dtype=torch.bfloat16, device="cuda").t(), w)
    with pytest.raises(ValueError):
        op.backward(x, w, x)
    with pytest.raises(ValueError):
        P.TokenNorm(4, 32, torch.bfloat16, kind="batch")
    with pytest.raises(TypeError):
        P.TokenNorm(4, 32, torch.float16)
    with pytest.raises(P.AgrlError):
        P.TokenNorm(4, 32, torch.bfloat16, eps=-1.0).forward(x, w)
