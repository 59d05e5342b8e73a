"""Packed causal attention, forward and backward, against its definition in 64 bits.

Bounds, with u = 2^-24 and r the type's half step (bf16 2^-8, fp32 u):
  S        products of d terms and the scale: e_S = (d + 8) u scale sum|q k|; the exponent is formed once
           from it and lse or the maximum, so P is off by e_P = e_S + (16 + |lse| + |S|) u of itself,
           and by r more where it is an operand
  o        sum P |v| (r + 2 e_P + n u) + r |o|       n: keys of the row (the sum's order)
  lse      max e_S + (n + 16 + 4 |lse|) u
  D        sum |do| (o's bound + d u |o|): the backward reads the o that the forward rounded
  dP       (d + 4) u sum |do v|
  dS       P (e_dP + e_D) + |dS| (e_P + r + 4 u) (a few u more where dP and D cancel: u P (|dP| + |D|))
  dv       sum P |do| (r + e_P + n u) + r |dv|       n: rows that are summed, over all heads of the group
  dq, dk   scale sum (e_dS + n u |dS|) |k or q| + r |dq|
"""
import numpy as np
import pytest
import torch

from helpers import log

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
BF, F32 = torch.bfloat16, torch.float32
HALF = {BF: 2.0 ** -8, F32: U}


def _np(t):
    return t.detach().double().cpu().numpy()


def _ref(q, k, v, off, do, scale, dtype):
    """(values, bounds) of o, lse, dq, dk, dv; [T, heads, d] arrays of doubles."""
    T, H, d = q.shape
    rep, r = H // k.shape[1], HALF[dtype]
    z = lambda *s: np.zeros(s)                                                    # noqa: E731
    val = dict(o=z(T, H, d), lse=z(H, T), dq=z(T, H, d), dk=z(*k.shape), dv=z(*k.shape))
    tol = {n: np.zeros_like(a) for n, a in val.items()}
    for b, e in zip(off, off[1:]):
        n = e - b
        if n <= 0:
            continue
        low = np.tril(np.ones((n, n), bool))
        for h in range(H):
            g, Q, D = h // rep, q[b:e, h], do[b:e, h]
            K, V = k[b:e, g], v[b:e, g]
            S = scale * (Q @ K.T)
            m = np.where(low, S, -np.inf).max(1, keepdims=True)
            P = np.where(low, np.exp(np.where(low, S, m) - m), 0.0)
            lse = m + np.log(P.sum(1, keepdims=True))
            P = np.where(low, np.exp(np.where(low, S, -np.inf) - lse), 0.0)
            eS = (d + 8) * U * scale * (np.abs(Q) @ np.abs(K).T)
            eP = np.where(low, eS + (16 + np.abs(lse) + np.abs(S)) * U, 0.0)
            cnt = np.arange(1, n + 1)[:, None]
            o = P @ V
            to = (P * (r + 2 * eP.max(1, keepdims=True) + cnt * U)) @ np.abs(V) + r * np.abs(o)
            val["o"][b:e, h], tol["o"][b:e, h] = o, to
            val["lse"][h, b:e] = lse[:, 0]
            tol["lse"][h, b:e] = (np.where(low, eS, 0).max(1) + (cnt[:, 0] + 16 + 4 * np.abs(lse[:, 0])) * U)
            dP, Dl = D @ V.T, (D * o).sum(1, keepdims=True)
            dS = P * (dP - Dl)
            eD = (np.abs(D) * (to + d * U * np.abs(o))).sum(1, keepdims=True)
            e_dS = (P * ((d + 4) * U * (np.abs(D) @ np.abs(V).T) + eD + U * (np.abs(dP) + np.abs(Dl)))
                    + np.abs(dS) * (eP + r + 4 * U))
            rows = rep * n
            val["dv"][b:e, g] += P.T @ D
            tol["dv"][b:e, g] += (P * (r + eP + rows * U)).T @ np.abs(D)
            val["dq"][b:e, h] = scale * dS @ K
            tol["dq"][b:e, h] = scale * (e_dS + n * U * np.abs(dS)) @ np.abs(K)
            val["dk"][b:e, g] += scale * dS.T @ Q
            tol["dk"][b:e, g] += scale * (e_dS + rows * U * np.abs(dS)).T @ np.abs(Q)
    for n in ("dq", "dk", "dv"):
        tol[n] += r * np.abs(val[n])
    return val, tol


def _make(T, H, G, d, dtype, seed=0, spread=1.5):
    g = torch.Generator().manual_seed(seed + 7919 * T + 31 * H + d)
    mk = lambda *s: torch.randn(*s, generator=g)                                  # noqa: E731
    q, k, v, do = spread * mk(T, H, d), mk(T, G, d) + 0.5 * mk(G, d), mk(T, G, d), 0.01 * mk(T, H, d)
    return [t.to(dtype) for t in (q, k, v, do)]


def _dead(T, off):
    dead = np.ones(T, bool)
    for b, e in zip(off, off[1:]):
        dead[b:e] = False
    return dead


def _check(got, val, tol, dead, what):
    share = {}
    for name, t in got.items():
        a, w, b = _np(t), val[name], tol[name]
        assert np.isfinite(a).all(), (what, name)
        share[name] = float((np.abs(a - w) / (b + 1e-30)).max(initial=0.0))
        z = a[:, dead] if name == "lse" else a[dead]
        assert not z.any() and not np.signbit(z).any(), (what, name, "tokens of no sequence")
    log("  shares of the bounds: " + " ".join(f"{n} {s:.2f}" for n, s in share.items()))
    assert max(share.values()) <= 1.0, (what, share)


def _offsets(off):
    return torch.tensor(off, dtype=torch.int32, device="cuda")


def _run(T, H, G, d, dtype, off, layout="fused", scale=None, seed=0, backward=True):
    import paper_2510_04206_amd as P
    log(f"attention T={T} heads {H}/{G} d={d} {dtype} seqs {len(off) - 1} {off[:6]} {layout}")
    q, k, v, do = _make(T, H, G, d, dtype, seed)
    dead = torch.from_numpy(_dead(T, off))
    for t in (q, k, v, do):                       # tokens of no sequence may hold anything
        t[dead] = float("nan")
    if layout == "fused":                         # parts of one projection's output
        qkv = torch.cat([q, k, v], 1).cuda()
        qd, kd, vd = qkv.split((H, G, G), 1)
        dod = do.cuda()
    elif layout == "heads first":
        qd, kd, vd, dod = (t.transpose(0, 1).contiguous().cuda().transpose(0, 1) for t in (q, k, v, do))
    elif layout == "odd":                         # any element, any pitch
        def odd(t):
            flat = torch.full((T * (t.shape[1] * d + 5) + 3,), float("nan"), dtype=dtype, device="cuda")
            w = flat[3:].as_strided(t.shape, (t.shape[1] * d + 5, d, 1))
            w.copy_(t)
            return w
        qd, kd, vd, dod = (odd(t) for t in (q, k, v, do))
    else:                                         # one key head for all, repeated by a stride of 0
        assert layout == "repeated"
        k, v = k[:, :1].expand(-1, G, -1), v[:, :1].expand(-1, G, -1)
        qd, dod = q.cuda(), do.cuda()
        kd, vd = (t[:, :1].contiguous().cuda().expand(-1, G, -1) for t in (k, v))
    s = d ** -0.5 if scale is None else scale
    op = P.PackedAttention(T, H, G, d, dtype, scale=scale, grads=backward)
    for t in (op.o, op.lse, op.dqkv):
        if t is not None:
            t.fill_(float("nan"))
    st = _offsets(off)
    o, lse = op.forward(qd, kd, vd, st)
    got = dict(o=o, lse=lse)
    if backward:
        got.update(zip(("dq", "dk", "dv"), op.backward(qd, kd, vd, st, dod)))
    torch.cuda.synchronize()
    assert P.agrl_get_device_error() == 0
    clean = lambda t: np.where(dead.numpy()[:, None, None], 0.0, _np(t))           # noqa: E731
    val, tol = _ref(clean(q), clean(k), clean(v), off, clean(do), s, dtype)
    _check(got, val, tol, dead.numpy(), (T, H, G, d, layout))
    return op


LENGTHS = [1, 2, 31, 32, 33, 63, 64, 65, 97, 127, 128, 129, 200, 257, 385]


@pytest.mark.parametrize("T", LENGTHS)
@pytest.mark.parametrize("dtype", [BF, F32])
def test_one_sequence(T, dtype):
    _run(T, 2, 1, 64, dtype, [0, T])


@pytest.mark.parametrize("d", [1, 3, 8, 17, 32, 33, 64, 65, 80, 96, 127, 128])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_head_sizes(d, dtype):
    _run(150, 3, 3, d, dtype, [0, 70, 150])


@pytest.mark.parametrize("H,G", [(1, 1), (4, 4), (8, 2), (7, 1), (10, 5), (28, 4), (40, 8)])
def test_shared_key_heads(H, G):
    _run(140, H, G, 64, BF, [0, 90, 140])


PACKINGS = {
    "edges": (400, [0, 32, 64, 127, 128, 129, 256, 321, 400]),
    "empty ones": (200, [0, 0, 5, 5, 5, 130, 130, 200, 200]),
    "padding": (300, [17, 40, 180, 263]),
    "all padding": (130, [50, 50]),
    "no sequence": (130, [3]),
    "ones": (200, list(range(201))),
    "sevens": (515, list(range(0, 512, 7))),
    "long and short": (640, [0, 500, 501, 503, 510, 640]),
}


@pytest.mark.parametrize("name", PACKINGS)
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
def test_packings(name, dtype, d):
    T, off = PACKINGS[name]
    _run(T, 4, 2, d, dtype, off)


@pytest.mark.parametrize("layout", ["heads first", "odd", "repeated"])
@pytest.mark.parametrize("d", [64, 100, 128])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_layouts(layout, d, dtype):
    _run(190, 4, 2, d, dtype, [0, 60, 188], layout)


@pytest.mark.parametrize("n_seq", [63, 64, 65, 4097, 5000])
def test_many_sequences(n_seq):
    """The search for a token's sequence takes 1, 2 and 3 steps of 64."""
    rng = np.random.default_rng(n_seq)
    off = np.concatenate([[0], np.cumsum(rng.integers(0, 3, n_seq))])
    _run(int(off[-1]) + 3, 2, 1, 64, BF, off.tolist())


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
def test_longer(dtype, d):
    """Several rounds of the pipelines, whole tiles among them."""
    _run(1200, 3, 1, d, dtype, [0, 700, 1190])


@pytest.mark.parametrize("scale", [1e-3, 3.0])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_scales(scale, dtype):
    """Nearly uniform rows, and rows of one key (maxima that move by hundreds)."""
    _run(300, 2, 2, 64, dtype, [0, 300], scale=scale)


def test_rising_scores():
    """Every tile's scores lie above the last one's: the softmax's reference moves in every step, and
    falling ones: it never does."""
    import paper_2510_04206_amd as P
    T, d = 520, 64
    for sign in (1.0, -1.0):
        log(f"attention rising {sign}")
        q = torch.zeros(T, 1, d)
        q[..., 0] = 8.0
        k = torch.zeros(T, 1, d)
        k[:, 0, 0] = sign * torch.arange(T) / 4
        k = k.to(BF).float()
        v = torch.randn(T, 1, d, generator=torch.Generator().manual_seed(1)).to(BF).float()
        op = P.PackedAttention(T, 1, 1, d, BF, scale=1.0, grads=False)
        o, lse = op.forward(q.to(BF).cuda(), k.to(BF).cuda(), v.to(BF).cuda(), _offsets([0, T]))
        zero = np.zeros((T, 1, d))
        val, tol = _ref(_np(q), _np(k), _np(v), [0, T], zero, 1.0, BF)
        _check(dict(o=o, lse=lse), val, tol, np.zeros(T, bool), sign)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_every_key_counts_once(dtype):
    """q = 0 and v a unit vector per key: o[n, j] = 1 / (n - begin + 1) for the keys of the row, else 0."""
    import paper_2510_04206_amd as P
    T, off = 128, [0, 50, 51, 128]
    log(f"attention weights {dtype}")
    q = torch.zeros(T, 1, 128, dtype=dtype, device="cuda")
    v = torch.eye(T, 128, device="cuda").to(dtype)[:, None]
    o, _ = P.PackedAttention(T, 1, 1, 128, dtype, grads=False).forward(q, torch.ones_like(q), v, _offsets(off))
    want = np.zeros((T, T))
    for b, e in zip(off, off[1:]):
        for n in range(b, e):
            want[n, b:n + 1] = 1.0 / (n - b + 1)
    # one rounding of the weight 1 (none), 1 / l and the result: 2 half steps and a few u
    assert (np.abs(_np(o)[:, 0] - want) <= (HALF[dtype] + 8 * U) * want).all()


def test_gradients_against_differences():
    """fp32, central differences of L = sum do o in one direction of each input.  A step h of 2^-6: the
    truncation is h^2 / 6 of the third derivative (measured on the 64-bit formula itself), the rounding
    of L (2^-24 of sum |do o|, a few hundred terms that mostly cancel) over 2 h."""
    import paper_2510_04206_amd as P
    T, H, G, d, off = 90, 4, 2, 64, [0, 40, 90]
    log("attention gradients against differences")
    q, k, v, do = _make(T, H, G, d, F32)
    do *= 100
    op = P.PackedAttention(T, H, G, d, F32)
    st = _offsets(off)
    fwd = lambda a, b, c: op.forward(a.cuda(), b.cuda(), c.cuda(), st)[0].double().cpu()     # noqa: E731
    fwd(q, k, v)
    grads = [g.double().cpu() for g in op.backward(q.cuda(), k.cuda(), v.cuda(), st, do.cuda())]
    h = 2.0 ** -6
    gen = torch.Generator().manual_seed(5)
    for i, x in enumerate((q, k, v)):
        w = torch.randn(x.shape, generator=gen)
        w /= w.norm()
        args = lambda s: [t + s * w if j == i else t for j, t in enumerate((q, k, v))]       # noqa: E731
        up, dn = ((fwd(*args(s)) * do.double()).sum() for s in (h, -h))
        got = float((grads[i] * w.double()).sum())
        loss = lambda s: (torch.from_numpy(_ref(*(_np(t) for t in args(s)), off, _np(do), d ** -0.5,   # noqa: E731
                                                F32)[0]["o"]) * do.double()).sum()
        exact = float((loss(h) - loss(-h)) / (2 * h))
        rounding = float((do.double().abs() * fwd(q, k, v).abs()).sum()) * (d + 64) * U / h
        assert abs(float((up - dn) / (2 * h)) - exact) <= rounding
        trunc = abs(exact - float((loss(h / 2) - loss(-h / 2)) / h)) * 2
        assert abs(got - exact) <= trunc + rounding, (i, got, exact)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
def test_masked_values_reach_no_one(bad, dtype, d):
    """One token's q, k, v and do are not finite: rows before it and other sequences keep their bits."""
    import paper_2510_04206_amd as P
    T, H, G, off, at = 300, 4, 2, [0, 110, 205, 300], 150
    log(f"attention masked {bad} {dtype} {d}")
    q, k, v, do = (t.cuda() for t in _make(T, H, G, d, dtype))
    op, st = P.PackedAttention(T, H, G, d, dtype), _offsets(off)
    run = lambda: [t.clone() for t in (*op.forward(q, k, v, st), *op.backward(q, k, v, st, do))]   # noqa: E731
    want = run()
    for t in (q, k, v, do):
        t[at] = bad
    got = run()
    other = [*range(0, 110), *range(205, 300)]
    early = [*range(0, at), *range(205, 300)]
    same = lambda a, b: torch.equal(a, b)                                          # noqa: E731
    assert same(got[0][early], want[0][early]) and same(got[1][:, early], want[1][:, early])
    for a, b in zip(got[2:], want[2:]):
        assert same(a[other], b[other])
    assert same(got[2][early], want[2][early])               # dq of rows that do not see the token
    assert not torch.isfinite(got[0][at:205].float()).any()  # and everyone who sees it is told
    assert not torch.isfinite(got[3][110:at + 1].float()).any() and not torch.isfinite(got[4][110:at + 1].float()).any()


def test_one_infinite_value_is_seen():
    """Only v is infinite, in a masked block: the rows that count it are not finite, no other changes."""
    import paper_2510_04206_amd as P
    T, d = 64, 64
    log("attention one infinite v")
    q, k, v, _ = (t.cuda() for t in _make(T, 1, 1, d, BF))
    op, st = P.PackedAttention(T, 1, 1, d, BF, grads=False), _offsets([0, T])
    want = op.forward(q, k, v, st)[0].clone()
    v[20, 0, 7] = float("inf")
    got = op.forward(q, k, v, st)[0]
    assert torch.equal(got[:20], want[:20])
    assert not torch.isfinite(got[20:, 0, 7].float()).any()
    keep = [c for c in range(d) if c != 7]
    assert torch.equal(got[20:, 0, keep], want[20:, 0, keep])


@pytest.mark.parametrize("dtype", [BF, F32])
def test_calls_repeat_their_bits(dtype):
    import paper_2510_04206_amd as P
    T, H, G, d = 700, 6, 2, 128
    log(f"attention repeat {dtype}")
    q, k, v, do = (t.cuda() for t in _make(T, H, G, d, dtype))
    op, st = P.PackedAttention(T, H, G, d, dtype), _offsets([0, 300, 690])
    run = lambda: [t.clone() for t in (*op.forward(q, k, v, st), *op.backward(q, k, v, st, do))]   # noqa: E731
    a, b = run(), run()
    assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_one_sequence_alone_or_packed():
    """A sequence between others has the results that it has alone, up to the bounds' roundings: the
    first row's exactly (its o is v, its dq and dk 0)."""
    import paper_2510_04206_amd as P
    T, H, G, d, off = 260, 2, 1, 64, [0, 61, 200, 260]
    log("attention first rows")
    q, k, v, do = (t.cuda() for t in _make(T, H, G, d, BF))
    op = P.PackedAttention(T, H, G, d, BF)
    st = _offsets(off)
    o, _ = op.forward(q, k, v, st)
    dq, dk, dv = op.backward(q, k, v, st, do)
    for b in off[:-1]:
        assert torch.equal(o[b], v[b].expand(H, d))
        assert not dq[b].any()
    one = P.PackedAttention(1, H, G, d, BF)
    o1, _ = one.forward(q[:1], k[:1], v[:1], _offsets([0, 1]))
    g1 = one.backward(q[:1], k[:1], v[:1], _offsets([0, 1]), do[:1])
    assert torch.equal(o1[0], o[0]) and not g1[0].any() and not g1[1].any()


def test_bad_offsets_set_the_error_bit():
    """Offsets out of order or range stay within the stream and are reported."""
    import paper_2510_04206_amd as P
    T = 100
    q, k, v, do = (t.cuda() for t in _make(T, 2, 1, 64, BF))
    for off in ([0, 60, 30, 100], [0, 50, 101], [-1, 40, 100], [100, 0]):
        log(f"attention offsets {off}")
        op = P.PackedAttention(T, 2, 1, 64, BF)
        op.forward(q, k, v, _offsets(off))
        assert P.agrl_get_device_error() == 32
        op.backward(q, k, v, _offsets(off), do)
        assert P.agrl_get_device_error() == 32
    op.forward(q, k, v, _offsets([0, 100]))
    assert P.agrl_get_device_error() == 0


def test_beyond_32_bits():
    """Rows whose elements lie past 2^31: the last tokens of a wide stream."""
    import paper_2510_04206_amd as P
    T, H, G, d = 140000, 128, 2, 128
    log("attention beyond 2^31 elements")
    off = [0, *range(100, T - 40, 100), T]
    q = torch.zeros(T, H, d, dtype=BF, device="cuda")
    do = torch.zeros_like(q)
    tail = slice(off[-2], T)
    n = T - off[-2]
    qs, ks, vs, dos = _make(n, H, G, d, BF)
    k, v = (torch.zeros(T, G, d, dtype=BF, device="cuda") for _ in range(2))
    for big, small in ((q, qs), (k, ks), (v, vs), (do, dos)):
        big[tail] = small.cuda()
    op = P.PackedAttention(T, H, G, d, BF)
    st = _offsets(off)
    o, lse = op.forward(q, k, v, st)
    dq, dk, dv = op.backward(q, k, v, st, do)
    hs = [0, 63, 64, 127]
    val, tol = _ref(_np(qs), _np(ks), _np(vs), [0, n], _np(dos), d ** -0.5, BF)
    got = dict(o=o[tail][:, hs], lse=lse[hs][:, tail], dq=dq[tail][:, hs], dk=dk[tail], dv=dv[tail])
    pick = lambda r: dict(o=r["o"][:, hs], lse=r["lse"][hs], dq=r["dq"][:, hs], dk=r["dk"], dv=r["dv"])   # noqa: E731
    _check(got, pick(val), pick(tol), np.zeros(n, bool), "tail")
    assert not dq[: off[-2]].any() and not dk[: off[-2]].any()


def test_captured_and_replayed():
    """Forward and backward in a graph, inputs changed between replays, eager calls of another handle in
    between: every replay has the eager bits."""
    import paper_2510_04206_amd as P
    T, H, G, d = 333, 4, 2, 64
    log("attention graph")
    st = _offsets([0, 100, 320])
    q, k, v, do = (t.cuda() for t in _make(T, H, G, d, BF))
    op, eager = P.PackedAttention(T, H, G, d, BF), P.PackedAttention(T, H, G, d, BF)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        op.forward(q, k, v, st)
        op.backward(q, k, v, st, do)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        op.forward(q, k, v, st)
        op.backward(q, k, v, st, do)
    for seed in range(4):
        for t, new in zip((q, k, v, do), _make(T, H, G, d, BF, seed=seed)):
            t.copy_(new)
        graph.replay()
        eager.forward(q, k, v, st)
        eager.backward(q, k, v, st, do)
        torch.cuda.synchronize()
        assert torch.equal(op.o, eager.o) and torch.equal(op.lse, eager.lse) and torch.equal(op.dqkv, eager.dqkv)
