"""Norms of rows with infinities, NaN, or squares beyond fp32's range: NaN as a whole, no other row."""
import pytest
import torch

from helpers import log

pytestmark = pytest.mark.gpu
# a length for each kind of team: one wave with one and two chunks, four, eight and sixteen waves
LENGTHS = [100, 513, 1025, 2049, 4097, 6145, 8193]


@pytest.mark.parametrize("d", LENGTHS)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_rows_out_of_range_are_nan(d, dtype, kind):
    import paper_2510_04206_amd as P
    log(f"norm rows out of range d={d} {dtype} {kind}")
    T = 23
    g = torch.Generator().manual_seed(d)
    x = torch.randn(T, d, generator=g).to(dtype).cuda()
    dy = torch.randn(T, d, generator=g).cuda()
    w, b = torch.randn(d, generator=g).cuda(), torch.randn(d, generator=g).cuda()
    op = P.TokenNorm(T, d, dtype, kind=kind)
    want = op.forward(x, w, b)[0].clone()
    want_dx = op.backward(x, w, dy)[0].clone()
    bad = {2: float("inf"), 5: float("-inf"), 9: float("nan"), 14: 3e19, 22: -3e38}
    for k, (row, value) in enumerate(bad.items()):
        x[row, (k * 37) % d] = value
    y, _, rstd = op.forward(x, w, b)
    dx = op.backward(x, w, dy)[0]
    rows = torch.zeros(T, dtype=torch.bool, device="cuda")
    rows[list(bad)] = True
    for got, ref in ((y, want), (dx, want_dx)):
        assert bool(torch.isnan(got[rows]).all())
        assert torch.equal(got[~rows], ref[~rows])
    assert bool(torch.isnan(rstd[rows]).all()) and bool(torch.isfinite(rstd[~rows]).all())
    # masked, they are not read
    mask = (~rows).to(torch.uint8)
    y = op.forward(x, w, b, mask)[0]
    dx, dw, db = op.backward(x, w, dy, mask)
    assert not y[rows].any() and not dx[rows].any() and torch.equal(y[~rows], want[~rows])
    assert bool(torch.isfinite(dw).all()) and (db is None or bool(torch.isfinite(db).all()))
