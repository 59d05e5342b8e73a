"""Rotation of heads by position, against the definition in 64 bits.

With u = 2^-24: the fraction of a turn is rounded to fp32 (2^-26 turns: 2 pi 2^-26 = 1.6 u), sine and cosine
to 2 units in the last place of at most 1 (2 u), the products and their sum 2 u: 8 u (|p| + |q|) with room; the 64-bit angle
itself is off by 4 2^-53 of its size.  Then one rounding to the type.
"""
import numpy as np
import pytest
import torch

from helpers import log

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
BF, F32 = torch.bfloat16, torch.float32


def _np(t):
    return t.detach().double().cpu().numpy()


def _ref(x, pos, rot, base, inter, inverse):
    y, tol = x.copy(), np.zeros_like(x)
    i = np.arange(rot // 2)
    ang = pos[:, None] * np.power(float(base), -2.0 * i / max(rot, 1))
    off = 8 * U + 4 * 2.0 ** -53 * np.abs(ang)[:, None, :]
    ang = (-ang if inverse else ang)[:, None, :]
    a, b = (slice(0, rot, 2), slice(1, rot, 2)) if inter else (slice(0, rot // 2), slice(rot // 2, rot))
    p, q = x[..., a], x[..., b]
    y[..., a], y[..., b] = p * np.cos(ang) - q * np.sin(ang), p * np.sin(ang) + q * np.cos(ang)
    tol[..., a] = tol[..., b] = off * (np.abs(p) + np.abs(q))
    return y, tol


def _run(T, H, d, rot, dtype, inter=False, inverse=False, base=1e4, pos="mixed", pitch=0, in_place=False):
    import paper_2510_04206_amd as P
    log(f"rotate T={T} heads={H} d={d} rot={rot} {dtype} inter {inter} inverse {inverse} {pos} pitch {pitch}")
    g = torch.Generator().manual_seed(T + 7 * H + d)
    x = torch.randn(T, H, d, generator=g).to(dtype)
    far = {"mixed": 1 << 20, "small": 300, "none": 0, "extreme": (1 << 31) - 1}[pos]
    p = torch.randint(-far, far + 1, (T,), generator=g).to(torch.int32)
    flat = torch.full((T, H * d + pitch), float("nan"), dtype=dtype, device="cuda")
    xd = flat[:, : H * d].unflatten(1, (H, d))
    xd.copy_(x)
    op = P.TokenRotation(T, H, d, dtype, rot=rot, base=base, interleaved=inter, output=not in_place)
    y = op(xd, None if pos == "none" else p.cuda(), inverse=inverse, out=xd if in_place else None)
    want, tol = _ref(_np(x), np.arange(T) * 1.0 if pos == "none" else _np(p), rot, base, inter, inverse)
    tol = tol + 1e-30 + (2.0 ** -8 * (np.abs(want) + tol) if dtype == BF else 0.0)
    share = float((np.abs(_np(y) - want) / tol).max())
    log(f"  share of the bound: {share:.2f}")
    assert share <= 1.0
    if rot < d:
        assert torch.equal(y[..., rot:].cpu(), x[..., rot:])
    if pitch:
        assert torch.isnan(flat[:, H * d:].float()).all()


@pytest.mark.parametrize("T,H,d,rot", [(1, 1, 2, 2), (1, 3, 64, 64), (150, 12, 64, 64), (33, 40, 128, 128), (7, 5, 34, 34),
                                       (9, 4, 96, 48), (20, 2, 80, 80), (5, 1, 33, 16), (3, 2, 512, 512), (4, 3, 300, 298),
                                       (700, 1, 16, 16), (6, 2, 8, 0), (4100, 2, 32, 32), (3, 300, 64, 64)])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("inter", [False, True])
def test_shapes(T, H, d, rot, dtype, inter):
    _run(T, H, d, rot, dtype, inter)
    _run(T, H, d, rot, dtype, inter, inverse=True, pitch=3)


@pytest.mark.parametrize("pos", ["small", "none", "extreme"])
@pytest.mark.parametrize("base", [1.0, 1e4, 1e6, 0.5])
def test_positions(pos, base):
    for dtype in (BF, F32):
        _run(90, 3, 64, 64, dtype, base=base, pos=pos)


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("rot", [128, 64, 30])
def test_in_place(inter, rot):
    for dtype in (BF, F32):
        _run(77, 6, 128, rot, dtype, inter, pitch=256, in_place=True)


def test_there_and_back():
    """inverse undoes the rotation: two roundings of each pair's bound, 16 u (|p| + |q|)."""
    import paper_2510_04206_amd as P
    T, H, d = 200, 4, 64
    x = torch.randn(T, H, d, device="cuda")
    pos = torch.arange(T, dtype=torch.int32, device="cuda") * 1000
    fwd, back = (P.TokenRotation(T, H, d, F32) for _ in range(2))
    y = back(fwd(x, pos), pos, inverse=True)
    pair = x[..., :32].abs() + x[..., 32:].abs()
    assert ((y - x).abs() <= 32 * U * torch.cat([pair, pair], 2)).all()


def test_beyond_32_bits():
    import paper_2510_04206_amd as P
    T, H, d = 140000, 128, 128
    log("rotate beyond 2^31 elements")
    x = torch.zeros(T, H, d, dtype=BF, device="cuda")
    x[-5:] = torch.randn(5, H, d, device="cuda").to(BF)
    op = P.TokenRotation(T, H, d, BF)
    y = op(x)
    want, tol = _ref(_np(x[-5:]), np.arange(T - 5, T) * 1.0, d, 1e4, False, False)
    assert (np.abs(_np(y[-5:]) - want) <= tol + 2.0 ** -8 * (np.abs(want) + tol) + 1e-30).all()
    assert not y[:-5].any()


def test_replays():
    import paper_2510_04206_amd as P
    T, H, d = 100, 5, 128
    log("rotate graph")
    x, pos = torch.randn(T, H, d, device="cuda"), torch.arange(T, dtype=torch.int32, device="cuda")
    op, eager = (P.TokenRotation(T, H, d, F32) for _ in range(2))
    op(x, pos)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        op(x, pos)
    for k in range(3):
        x.normal_()
        pos.add_(1000 * k)
        graph.replay()
        eager(x, pos)
        torch.cuda.synchronize()
        assert torch.equal(op.out, eager.out)
