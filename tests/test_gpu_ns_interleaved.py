"""Stacks whose matrices' rows take turns in memory: [m, batch, n] seen as [batch, m, n].  The same bits
as from a contiguous stack, and nothing written beside it."""
import pytest
import torch

from helpers import log

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def _turns(t, pad):
    """t's values with rows in turn, each row `pad` elements from the next one; and the whole buffer."""
    b, m, n = t.shape
    wide = torch.full((m, b, n + pad), 7.0, dtype=t.dtype, device="cuda")
    view = wide[..., :n].transpose(0, 1)
    view.copy_(t)
    return view, wide


@pytest.mark.parametrize("m,n", [(40, 90), (90, 41), (128, 300), (130, 201), (333, 150)])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("pad", [0, 5])
def test_muon(m, n, dtype, pad):
    import paper_2510_04206_amd as P
    log(f"muon of rows in turn, 3 x {m} x {n} {dtype} pad {pad}")
    g = torch.Generator().manual_seed(m)
    w = torch.randn(3, m, n, generator=g).to(dtype).cuda()
    grad = torch.randn(3, m, n, generator=g).cuda()
    mom = torch.zeros(3, m, n, device="cuda")
    op = P.MuonStep(m, n, param_dtype=dtype, batch=3, weight_decay=0.1)
    view, wide = _turns(w, pad)
    gview, _ = _turns(grad, pad)
    mom2 = mom.clone()
    op(w, grad, mom, 0.1)
    op(view, gview, mom2, 0.1)
    assert torch.equal(view, w) and torch.equal(mom2, mom)
    assert bool((wide[..., n:] == 7.0).all())


def test_overlapping_rows_are_refused():
    import paper_2510_04206_amd as P
    x = torch.zeros(8, 16, device="cuda")
    op = P.MuonStep(8, 16, batch=3)
    with pytest.raises(P.AgrlError):
        op(x.expand(3, 8, 16), torch.zeros(3, 8, 16, device="cuda"), torch.zeros(3, 8, 16, device="cuda"), 0.1)
