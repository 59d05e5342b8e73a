"""Embedding of packed tokens and its gradient, against the definition.

Forward: the weight in fp32 times the scale, rounded to fp32 and to the type: exact.  Gradient: a sum of n
terms in fp32 in a fixed order (pieces of 32, then the pieces), the scale and the addition: off by at most
(n + 4) u sum |dy| |scale| + u |dW before|, u = 2^-24.
"""
import numpy as np
import pytest
import torch

from helpers import log

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
BF, F32 = torch.bfloat16, torch.float32


def _ids(T, V, seed=0, kind="text"):
    rng = np.random.default_rng([seed, T, V])
    if kind == "same":
        ids = np.full(T, V // 2)
    elif kind == "all":
        ids = np.arange(T) * 7 % V
    else:
        ids = np.minimum((V * rng.random(T) ** 4).astype(np.int64), V - 1)
        ids = np.where(rng.random(T) < 0.2, V - 1, ids)
    return torch.from_numpy(ids.astype(np.int32))


def _mask(T, kind):
    if kind == "none":
        return None
    m = torch.zeros(T, dtype=torch.uint8)
    if kind == "some":
        m[torch.rand(T, generator=torch.Generator().manual_seed(T)) < 0.7] = 1
    return m


@pytest.mark.parametrize("T,d,V", [(1, 1, 1), (1, 5, 3), (3, 257, 50), (97, 256, 4096), (300, 1001, 70),
                                   (64, 2048, 33), (50, 2049, 33), (5, 8195, 10), (2000, 72, 5000)])
@pytest.mark.parametrize("wt,dt", [(BF, BF), (BF, F32), (F32, BF), (F32, F32)])
@pytest.mark.parametrize("mask", ["none", "some"])
def test_forward(T, d, V, wt, dt, mask):
    import paper_2510_04206_amd as P
    log(f"embed fwd T={T} d={d} V={V} {wt} {dt} {mask}")
    w = torch.randn(V, d, generator=torch.Generator().manual_seed(1)).to(wt)
    ids, m = _ids(T, V), _mask(T, mask)
    scale = 1.0 if T % 2 else d ** 0.5
    live = torch.ones(T, dtype=torch.bool) if m is None else m.bool()
    given = torch.where(live, ids, torch.full_like(ids, -5))      # a dead token's id is not read
    op = P.TokenEmbedding(T, V, d, dt, w_dtype=wt, scale=scale, grads=False)
    op.y.fill_(float("nan"))
    y = op.forward(w.cuda(), given.cuda(), None if m is None else m.cuda()).cpu()
    want = (w.float()[ids.long()] * torch.tensor(scale, dtype=F32)).to(dt)
    want[~live] = 0
    assert torch.equal(y, want) and not torch.signbit(y[~live]).any()
    assert P.agrl_get_device_error() == 0


def _grad(T, d, V, dt, kind="text", mask="none", accumulate=False, pitch=0, scale=1.0):
    import paper_2510_04206_amd as P
    log(f"embed bwd T={T} d={d} V={V} {dt} {kind} {mask} accumulate {accumulate} pitch {pitch}")
    g = torch.Generator().manual_seed(T + d)
    ids, m = _ids(T, V, kind=kind), _mask(T, mask)
    live = torch.ones(T, dtype=torch.bool) if m is None else m.bool()
    dy = torch.randn(T, d, generator=g).to(dt)
    wide = torch.full((T, d + pitch), float("nan"), dtype=dt, device="cuda")
    wide[:, :d] = dy.cuda()
    wide[:, :d][~live.cuda()] = float("nan")
    before = torch.randn(V, d, generator=g) if accumulate else torch.full((V, d), float("nan"))
    dw = before.cuda()
    op = P.TokenEmbedding(T, V, d, dt, scale=scale, dweight=dw)
    op.workspace.fill_(0xff)
    got = op.backward(torch.where(live, ids, torch.full_like(ids, V + 9)).cuda(), wide[:, :d],
                      None if m is None else m.cuda(), accumulate=accumulate)
    assert got is dw and P.agrl_get_device_error() == 0
    want = torch.zeros(V, d, dtype=torch.float64)
    size = torch.zeros(V, d, dtype=torch.float64)
    n = torch.zeros(V, dtype=torch.float64)
    li, ld = ids.long()[live], dy.double()[live] * scale
    want.index_add_(0, li, ld)
    size.index_add_(0, li, ld.abs())
    n.index_add_(0, li, torch.ones(len(li), dtype=torch.float64))
    if accumulate:
        want += before.double()
        size += before.double().abs()
        assert torch.equal(dw.cpu()[n == 0], before[n == 0])
    tol = (n[:, None] + 4) * U * size
    off = (dw.cpu().double() - want).abs()
    assert (off <= tol).all(), float((off / (tol + 1e-30)).max())
    return op


@pytest.mark.parametrize("T,d,V", [(1, 1, 1), (1, 7, 3), (2, 3, 2), (31, 64, 40), (32, 65, 40), (33, 1024, 40),
                                   (64, 1025, 7), (257, 1001, 4096), (3823, 130, 300), (1500, 40, 140000),
                                   (700, 5120, 1000)])
@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("accumulate", [False, True])
def test_gradient(T, d, V, dt, accumulate):
    _grad(T, d, V, dt, accumulate=accumulate, scale=1.0 if d % 2 else d ** 0.5)


@pytest.mark.parametrize("kind", ["same", "all", "text"])
@pytest.mark.parametrize("mask", ["some", "dead"])
def test_gradient_runs(kind, mask):
    """One id over all chunks, ids that hardly repeat, a text's; a mask that leaves some or none."""
    for T in (40, 1000, 5000):
        _grad(T, 33, 513, F32, kind=kind, mask=mask, pitch=3)
        _grad(T, 96, 100, BF, kind=kind, mask=mask, accumulate=True, pitch=5)


def test_no_tokens():
    import paper_2510_04206_amd as P
    op = P.TokenEmbedding(0, 50, 16, F32)
    op.dweight.fill_(3.0)
    empty = torch.zeros(0, dtype=torch.int32, device="cuda")
    op.backward(empty, torch.zeros(0, 16, device="cuda"), accumulate=True)
    assert (op.dweight == 3).all()
    op.backward(empty, torch.zeros(0, 16, device="cuda"))
    assert not op.dweight.any()
    assert op.forward(torch.zeros(50, 16, device="cuda"), empty).shape == (0, 16)


def test_ids_out_of_range():
    import paper_2510_04206_amd as P
    T, V, d = 200, 60, 40
    w, dy = torch.randn(V, d, device="cuda"), torch.randn(T, d, device="cuda")
    for bad in (-1, V, 2 ** 31 - 1, -2 ** 31):
        log(f"embed id {bad}")
        ids = _ids(T, V)
        ids[77] = bad
        op = P.TokenEmbedding(T, V, d, F32)
        y = op.forward(w, ids.cuda()).clone()
        assert P.agrl_get_device_error() == 1
        assert torch.isnan(y[77]).all()
        keep = [i for i in range(T) if i != 77]
        assert torch.equal(y[keep].cpu(), w.cpu()[ids[keep].long()])
        got = op.backward(ids.cuda(), dy).clone()
        assert P.agrl_get_device_error() == 1
        mask = torch.ones(T, dtype=torch.uint8)
        mask[77] = 0
        assert torch.equal(got, op.backward(ids.cuda(), dy, mask.cuda()))
        assert P.agrl_get_device_error() == 0


def test_nan_stays_in_its_row():
    import paper_2510_04206_amd as P
    T, V, d = 300, 40, 64
    ids, dy = _ids(T, V).cuda(), torch.randn(T, d, device="cuda")
    op = P.TokenEmbedding(T, V, d, F32)
    want = op.backward(ids, dy).clone()
    dy[100] = float("nan")
    got = op.backward(ids, dy)
    hit = int(ids[100])
    keep = [v for v in range(V) if v != hit]
    assert torch.isnan(got[hit]).all() and torch.equal(got[keep], want[keep])


def test_repeats_and_replays():
    """The gradient's bits do not change from call to call, nor in a graph whose inputs change."""
    import paper_2510_04206_amd as P
    T, V, d = 3000, 500, 256
    log("embed graph")
    ids, dy = _ids(T, V).cuda(), torch.randn(T, d, device="cuda").to(BF)
    w = torch.randn(V, d, device="cuda").to(BF)
    op, eager = P.TokenEmbedding(T, V, d, BF), P.TokenEmbedding(T, V, d, BF)
    a = op.backward(ids, dy).clone()
    assert torch.equal(a, op.backward(ids, dy))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        op.forward(w, ids)
        op.backward(ids, dy)
    for seed in range(4):
        ids.copy_(_ids(T, V, seed))
        dy.copy_(torch.randn(T, d, device="cuda"))
        graph.replay()
        eager.forward(w, ids)
        eager.backward(ids, dy)
        torch.cuda.synchronize()
        assert torch.equal(op.y, eager.y) and torch.equal(op.dweight, eager.dweight)


def test_beyond_32_bits():
    """A [V, d] of more than 2^31 elements, its last rows hit and cleared."""
    import paper_2510_04206_amd as P
    T, V, d = 64, 300000, 8192
    log("embed beyond 2^31 elements")
    ids = (V - 1 - torch.arange(T, dtype=torch.int32) // 2 * 3).cuda()
    dy = torch.randn(T, d, device="cuda")
    dw = torch.full((V, d), float("nan"), device="cuda")
    op = P.TokenEmbedding(T, V, d, F32, dweight=dw)
    op.backward(ids, dy)
    want = dy.view(T // 2, 2, d).sum(1)
    assert torch.equal(dw[ids[::2].long()], want)
    dw[ids.long()] = 0
    assert not dw[V - 2000:].any() and not dw[:2000].any() and not dw[V // 2: V // 2 + 2000].any()
    y = P.TokenEmbedding(T, V, d, F32, grads=False).forward(dw.copy_(torch.ones((), device="cuda")), ids)
    assert (y == 1).all()
