"""Norms of so many rows that a team goes through more than one group of 64, against the formula in 64 bits.

A forward team of 256 compute units' grid has its second group past 262144 rows (d <= 1024), 65536 (d <=
6144), 32768 (d <= 8192) or 16384 rows; the backward's past 131072 (d <= 1024) or 32768.  Bounds as in
test_gpu_norm.py, u = 2^-24: rstd 64 u; y 64 u (|w| (|xh| + X) + |b|); dx 128 u rstd (|g| + mean|g| +
(|xh| + X) mean|g xh|), and 2^-8 of the value for a bf16 one; dw (128 + T / 512 + 32) u sum |dy| (|xh| + X).
"""
import pytest
import torch

from helpers import log

pytestmark = pytest.mark.gpu
U, EPS = 2.0 ** -24, 1e-5


def _near(got, want, tol, what):
    tol = tol + 1e-30 + (2.0 ** -8 * want.abs() if got.dtype == torch.bfloat16 else 0.0)
    off = (got.double() - want).abs()
    assert bool(torch.isfinite(got).all()) and bool((off <= tol).all()), (what, float((off / tol).max()))


def _rows(x, live, w, b, kind):
    """mean, rstd, xh and max |x| rstd of the rows, in 64 bits; 0 where masked."""
    x = torch.where(live[:, None], x.double(), 0.0)
    mean = x.mean(1) if kind == "layer" else torch.zeros_like(x[:, 0])
    xc = x - mean[:, None]
    rstd = torch.where(live, ((xc * xc).mean(1) + EPS) ** -0.5, 0.0)
    return x, mean, rstd, xc * rstd[:, None], (x.abs().amax(1) * rstd)[:, None]


# one wave with one and two chunks, four waves, eight, sixteen; past the second group's end for some teams
@pytest.mark.parametrize("T,d,backward", [
    (263000, 8, True), (270001, 520, True), (530000, 16, False), (66001, 1032, True), (140003, 1030, False),
    (66003, 2056, True), (66005, 4100, False), (33001, 6152, True), (16501, 8200, False), (33003, 8200, True)])
@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("masked", [False, True])
def test_more_than_a_group(T, d, backward, kind, masked):
    import paper_2510_04206_amd as P
    log(f"norm T={T} d={d} backward {backward} {kind} masked {masked}")
    g = torch.Generator(device="cuda").manual_seed(T + d)
    randn = lambda *n: torch.randn(*n, generator=g, device="cuda")                # noqa: E731
    x = (randn(T, d) * torch.exp(randn(T, 1)) + 0.3).bfloat16()
    w, b = 1 + 0.3 * randn(d), 0.3 * randn(d)
    live = torch.rand(T, generator=g, device="cuda") < 0.4 if masked else torch.ones(T, device="cuda").bool()
    live[-1] = True
    mask = live.to(torch.uint8) if masked else None
    op = P.TokenNorm(T, d, torch.bfloat16, kind=kind, eps=EPS, grads=backward, bias_grad=True)
    for t in op._buffers:
        if t.dtype.is_floating_point:
            t.fill_(float("nan"))
    y, mean, rstd = op.forward(x, w, b, mask)
    if backward:
        dy = 0.01 * randn(T, d)
        dx, dw, db = op.backward(x, w, dy, mask)
        sums = [torch.zeros(d, dtype=torch.float64, device="cuda") for _ in range(4)]
    w64, b64 = w.double(), b.double()
    for r in range(0, T, 16384):                             # (the reference by parts: memory)
        s = slice(r, min(r + 16384, T))
        lv = live[s]
        x64, m64, r64, xh, X = _rows(x[s], lv, w64, b64, kind)
        near = torch.where(lv[:, None], xh * w64 + b64, 0.0)
        _near(y[s], near, 64 * U * (w64.abs() * (xh.abs() + X) + b64.abs()), "y")
        _near(rstd[s], r64, 64 * U * r64, "rstd")
        if kind == "layer":
            _near(mean[s], m64, 64 * U * x64.abs().amax(1), "mean")
        if not backward:
            continue
        dy64 = torch.where(lv[:, None], dy[s].double(), 0.0)
        gr = dy64 * w64
        c1 = gr.mean(1, keepdim=True) if kind == "layer" else 0.0
        want = r64[:, None] * (gr - c1 - xh * (gr * xh).mean(1, keepdim=True))
        tol = 128 * U * r64[:, None] * (gr.abs() + gr.abs().mean(1, keepdim=True) +
                                        (xh.abs() + X) * (gr * xh).abs().mean(1, keepdim=True))
        _near(dx[s], want, tol, "dx")
        for t, v in zip(sums, (dy64 * xh, dy64, dy64.abs() * (xh.abs() + X), dy64.abs())):
            t += v.sum(0)
    if backward:
        n = 128 + -(-T // 512) + 32
        _near(dw, sums[0], n * U * sums[2], "dw")
        _near(db, sums[1], n * U * sums[3], "db")
