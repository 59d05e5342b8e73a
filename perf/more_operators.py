"""The operators between the token ids and the final norm that are timed.

Five calls, each as a trainer on packed trajectories meets it:

  emb_fwd   rows of the embedding for a packed stream of token ids (``TokenEmbedding.forward``);
  emb_bwd   the embedding's gradient, rows added up by token id, into a new [V, d] or onto one
            that the head's gradient is in already (``TokenEmbedding.backward``);
  rotate    position rotation of the query and key heads inside a fused projection, positions
            counted from each trajectory's start (``TokenRotation``);
  att_fwd   causal attention within each trajectory of the stream, query heads sharing key
            heads (``PackedAttention.forward``);
  att_bwd   its gradients (``PackedAttention.backward``).

``run`` computes either the plain form in 32 bits with elementary torch operations, or calls
the framework (``own``); ``exact`` computes the definitions in 64 bits.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BYTES = {"bf16": 2, "f32": 4}


# ------------------------------------------------------------------ the cases
def listed():
    emb = dict(dtype="bf16", wdtype="bf16", scale=1.0, masked=False)
    bwd = dict(op="emb_bwd", dtype="bf16", scale=1.0, masked=False, accumulate=False, pitch=0)
    rot = dict(op="rotate", dtype="bf16", base=1e6, interleaved=False, inverse=False, far=0)
    att = dict(dtype="bf16", d=128)
    return [
        # a short turn in a toy model: launch and latency
        dict(emb, op="emb_fwd", name="embed fwd short turn", T=97, d=256, V=4096, wdtype="f32", dtype="f32"),
        # the 32B-shaped micro-batch, looked up in a bf16 embedding
        dict(emb, op="emb_fwd", name="embed fwd 64k", T=65536, d=5120, V=152064),
        # a small model of odd width, padded rows, the head's gradient already in the buffer
        dict(bwd, name="embed bwd odd tied", T=3823, d=1001, V=4096, masked=True, accumulate=True,
             scale=31.0, dtype="f32", pitch=7),
        # the 32B-shaped micro-batch: a whole [V, d] gradient out of 64k rows
        dict(bwd, name="embed bwd 64k", T=65536, d=5120, V=152064),
        # one turn's queries and keys in a toy model in fp32, neighbouring elements paired
        dict(rot, name="rotate short turn", T=150, heads=12, skip=6, d=64, rot=64, dtype="f32",
             kind="one", interleaved=True, base=1e4),
        # queries and keys of the 64k micro-batch inside the fused projection's output
        dict(rot, name="rotate 64k", T=65536, heads=48, skip=8, d=128, rot=128, kind="turns"),
        # a short turn: one sequence, few heads
        dict(att, op="att_fwd", name="attention fwd short turn", T=97, heads=8, kv=2, d=64, kind="one"),
        # the 7B-shaped micro-batch: whole trajectories end to end
        dict(att, op="att_fwd", name="attention fwd packed 32k", T=32768, heads=28, kv=4, kind="turns"),
        # long horizon: trajectories of tens of turns
        dict(att, op="att_fwd", name="attention fwd long horizon", T=32768, heads=40, kv=8, kind="long"),
        # a debugging run's whole micro-batch in fp32
        dict(att, op="att_bwd", name="attention bwd toy f32", T=1519, heads=4, kv=2, d=64, dtype="f32",
             kind="short"),
        # single turns of a few tokens, some empty, padding behind the last; odd head size
        dict(att, op="att_bwd", name="attention bwd ragged", T=8191, heads=16, kv=4, d=80, kind="short"),
        # half of the 7B-shaped micro-batch
        dict(att, op="att_bwd", name="attention bwd packed 16k", T=16384, heads=28, kv=4, kind="turns"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """Log-uniform; half of them odd or otherwise ragged, the others multiples of 64."""
    v = _log(rng, lo, hi)
    return v // 64 * 64 if rng.random() < 0.5 and v >= 64 else v


def draw(rng):
    op = rng.choice(["emb_fwd", "emb_bwd", "rotate", "att_fwd", "att_bwd"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    kind = rng.choice(["one", "turns", "long", "short"])
    if op.startswith("emb"):
        T, d, V = _log(rng, 1, 131072), _width(rng, 64, 8192), _log(rng, 500, 160000)
        T, V = max(1, min(T, 65536 * 5120 // d)), max(2, min(V, 152064 * 5120 // d))
        c = dict(op=op, T=T, d=d, V=V, dtype=dtype, scale=rng.choice([1.0, 1.0, math.sqrt(d)]),
                 masked=rng.random() < 0.3)
        if op == "emb_fwd":
            c["wdtype"] = rng.choice(["bf16", "f32"])
        else:
            c.update(accumulate=rng.random() < 0.5, pitch=rng.choice([0, 0, 64, 5]))
        return c
    if op == "rotate":
        d = rng.choice([64, 128, 128, 96, 80, 34])
        heads = rng.choice([1, 5, 12, 32, 48])
        T = max(1, min(_log(rng, 1, 131072), 65536 * 48 * 128 // (heads * d)))
        return dict(op=op, T=T, heads=heads, skip=rng.choice([0, 2, 8]), d=d,
                    rot=rng.choice([d, d, d // 4 * 2]), dtype=dtype, base=rng.choice([1e4, 1e6]),
                    interleaved=rng.random() < 0.3, inverse=rng.random() < 0.4,
                    far=rng.choice([0, 0, 1 << 20]), kind=kind)
    kv = rng.choice([1, 2, 4, 8])
    heads = kv * rng.choice([1, 1, 2, 5, 7]) if kv < 8 else kv * rng.choice([1, 4, 5])
    c = dict(op=op, T=_log(rng, 1, 32768), heads=heads, kv=kv, d=rng.choice([64, 128, 128, 128, 96, 80, 33]),
             dtype=dtype, kind=kind)
    most = _largest_attention()
    while work(c)["flops"] * (4 if dtype == "f32" else 1) > most:
        c["T"] = c["T"] * 3 // 4
    return c


def _largest_attention():
    return max(work(c)["flops"] for c in listed() if c["op"] in ("att_fwd", "att_bwd"))


# ------------------------------------------------------------------ inputs
def _offsets(c):
    """Ends of the sequences of a stream of T tokens, from 0: the packing is the case's."""
    T, rng = c["T"], np.random.default_rng([c["T"], 11])
    if c["kind"] == "one":
        return [0, T]
    if c["kind"] == "short":          # single turns, now and then an empty one, a little padding behind
        n = T // 32 + 1
        lens = np.where(rng.random(n) < 0.05, 0, rng.integers(1, 65, n))
        end, cut = np.cumsum(lens), T - T // 100
        return [0] + [int(min(e, cut)) for e in end]
    turns = (30, 50) if c["kind"] == "long" else (4, 12)
    off = [0]
    while off[-1] < T:                # turns of observation and action tokens; the last one is cut
        n = int(rng.integers(turns[0], turns[1] + 1))
        obs, act = ((128, 1025), (16, 129)) if c["kind"] == "long" else ((64, 513), (32, 257))
        off.append(min(T, off[-1] + int(rng.integers(*obs, n).sum() + rng.integers(*act, n).sum())))
    return off


def _positions(c):
    """Each token's position in its trajectory (behind the last one: counted on)."""
    off = np.asarray(_offsets(c))
    t = np.arange(c["T"])
    return (t - off[np.clip(np.searchsorted(off, t, side="right") - 1, 0, None)] + c["far"]).astype(np.int32)


def _ids(T, V, seed):
    """Token ids as text has them: a few separators everywhere, the rest by frequency."""
    rng = np.random.default_rng([seed, 5])
    ids = np.minimum((V * rng.random(T) ** 4).astype(np.int64), V - 1)
    ids = np.where(rng.random(T) < 0.12, rng.integers(0, 4, T) * (V // 4), ids)
    return torch.from_numpy(ids.astype(np.int32)).to(DEV)


def _wide(t, pitch):
    """The same rows in a buffer that is `pitch` elements wider."""
    if not pitch:
        return t
    wide = torch.zeros(t.shape[0], t.shape[1] + pitch, dtype=t.dtype, device=t.device)
    wide[:, : t.shape[1]] = t
    return wide[:, : t.shape[1]]


def prepare(case, seed):
    c, g = case, torch.Generator(device=DEV).manual_seed(seed)
    s, T, d, dt = dict(case=c), c["T"], c["d"], DTYPES[c["dtype"]]
    randn = lambda *n, dtype=torch.float32: torch.randn(*n, generator=g, device=DEV, dtype=dtype)  # noqa: E731
    if c["op"].startswith("emb"):
        s["ids"] = _ids(T, c["V"], seed)
        s["live"] = None
        if c["masked"]:               # padding at the end and now and then within
            live = np.random.default_rng([seed, 6]).random(T) > 0.05
            live[T - T // 50:] = False
            s["live"] = torch.from_numpy(live.astype(np.uint8)).to(DEV)
        if c["op"] == "emb_fwd":
            s["weight"] = randn(c["V"], d, dtype=DTYPES[c["wdtype"]]).mul_(0.02)
        else:
            s["dy"] = _wide(randn(T, d).mul_(1e-2).to(dt), c["pitch"])
            if c["accumulate"]:
                s["dweight"] = randn(c["V"], d).mul_(1e-2)
    elif c["op"] == "rotate":
        s["x"] = randn(T, c["heads"] + c["skip"], d, dtype=dt)[:, : c["heads"]]
        s["position"] = torch.from_numpy(_positions(c)).to(DEV)
    else:
        h, kv = c["heads"], c["kv"]
        # a fused projection's output; keys with an offset, so that some weights stand out
        qkv = randn(T, h + 2 * kv, d)
        qkv[:, :h] *= 1.5
        qkv[:, h:h + kv] += 0.5 * randn(kv, d)
        qkv = qkv.to(dt)
        s["q"], s["k"], s["v"] = qkv[:, :h], qkv[:, h:h + kv], qkv[:, h + kv:]
        s["off"] = _offsets(c)
        s["seq_start"] = torch.tensor(s["off"], dtype=torch.int32, device=DEV)
        if c["op"] == "att_bwd":
            s["do"] = randn(T, h, d).mul_(1e-2).to(dt)
            s["o"], s["lse"] = _plain_att_fwd(s)                 # what the forward left
    if own:
        # the handle a program keeps: workspace and outputs of one shape
        import paper_2510_04206_amd as P
        if c["op"] == "emb_fwd":
            s["op"] = P.TokenEmbedding(T, c["V"], d, dt, w_dtype=DTYPES[c["wdtype"]], scale=c["scale"],
                                       grads=False, device=DEV)
        elif c["op"] == "emb_bwd":
            s["op"] = P.TokenEmbedding(T, c["V"], d, dt, scale=c["scale"], dweight=s.get("dweight"), device=DEV)
        elif c["op"] == "rotate":
            s["op"] = P.TokenRotation(T, c["heads"], d, dt, rot=c["rot"], base=c["base"],
                                      interleaved=c["interleaved"], device=DEV)
        else:
            s["op"] = P.PackedAttention(T, c["heads"], c["kv"], d, dt, grads=c["op"] == "att_bwd", device=DEV)
            if c["op"] == "att_bwd":
                s["op"].o.copy_(s["o"])
                s["op"].lse.copy_(s["lse"])
    return s


# ------------------------------------------------------------------ one pass
def run(s):
    op = s["case"]["op"]
    if own:
        return _run_own(s)
    return {"emb_fwd": _plain_emb_fwd, "emb_bwd": _plain_emb_bwd, "rotate": _plain_rotate,
            "att_fwd": _plain_att_fwd, "att_bwd": _plain_att_bwd}[op](s)


def _run_own(s):
    c, call = s["case"], s["op"]
    if c["op"] == "emb_fwd":
        return [call.forward(s["weight"], s["ids"], s["live"])]
    if c["op"] == "emb_bwd":
        return [call.backward(s["ids"], s["dy"], s["live"], accumulate=c["accumulate"])]
    if c["op"] == "rotate":
        return [call(s["x"], s["position"], inverse=c["inverse"])]
    if c["op"] == "att_fwd":
        return list(call.forward(s["q"], s["k"], s["v"], s["seq_start"]))
    return list(call.backward(s["q"], s["k"], s["v"], s["seq_start"], s["do"]))


def _plain_emb_fwd(s):
    y = s["weight"][s["ids"].long()].float() * s["case"]["scale"]
    if s["live"] is not None:
        y = y * s["live"][:, None]
    return [y.to(DTYPES[s["case"]["dtype"]])]


def _plain_emb_bwd(s):
    c, ids, dy = s["case"], s["ids"].long(), s["dy"].float() * s["case"]["scale"]
    if s["live"] is not None:
        dy = dy * s["live"][:, None]
    dw = s["dweight"] if c["accumulate"] else torch.zeros(c["V"], c["d"], device=DEV)
    return [dw.index_add_(0, ids, dy)]


def _turn(s, real):
    """cos and sin of every token's angles, [T, 1, rot / 2], the angles in 64 bits."""
    c = s["case"]
    i = torch.arange(c["rot"] // 2, dtype=torch.float64, device=DEV)
    a = s["position"].double()[:, None] * torch.exp(i * (-2.0 / max(c["rot"], 1) * math.log(c["base"])))
    a = (-a if c["inverse"] else a)[:, None, :]
    return torch.cos(a).to(real), torch.sin(a).to(real)


def _plain_rotate(s):
    c, x = s["case"], s["x"].float()
    r, (cos, sin) = c["rot"], _turn(s, torch.float32)
    y = x.clone()
    a, b = (slice(0, r, 2), slice(1, r, 2)) if c["interleaved"] else (slice(0, r // 2), slice(r // 2, r))
    y[..., a] = x[..., a] * cos - x[..., b] * sin
    y[..., b] = x[..., a] * sin + x[..., b] * cos
    return [y.to(s["x"].dtype)]


def _pieces(s):
    """(sequence, key head, query heads at a time) whose score matrices fit a few GiB."""
    c = s["case"]
    rep = c["heads"] // c["kv"]
    for b, e in zip(s["off"], s["off"][1:]):
        at_once = max(1, (1 << 30) // max(1, (e - b) ** 2))
        if e > b and at_once >= c["heads"]:
            yield b, e, slice(0, c["kv"]), slice(0, c["heads"])
        elif e > b:
            for h in range(c["heads"]):
                yield b, e, slice(h // rep, h // rep + 1), slice(h, h + 1)


def _heads(t, b, e, hs, n=1):
    """[heads, tokens, d] of a piece in fp32, each head n times in turn."""
    x = t[b:e, hs].float().transpose(0, 1)
    return (x[:, None].expand(-1, n, -1, -1).reshape(-1, *x.shape[1:]) if n > 1 else x).contiguous()


def _plain_att_fwd(s):
    c, scale = s["case"], s["case"]["d"] ** -0.5
    o = torch.zeros(c["T"], c["heads"], c["d"], device=DEV, dtype=s["q"].dtype)
    lse = torch.zeros(c["heads"], c["T"], device=DEV)
    for b, e, ks, hs in _pieces(s):
        n = (hs.stop - hs.start) // (ks.stop - ks.start)
        q, k, v = _heads(s["q"], b, e, hs), _heads(s["k"], b, e, ks, n), _heads(s["v"], b, e, ks, n)
        p = torch.matmul(q, k.transpose(1, 2).contiguous()).mul_(scale)
        i = torch.arange(e - b, device=DEV)
        p.masked_fill_(i[None, :] > i[:, None], -math.inf)
        m = p.amax(2, keepdim=True)
        p.sub_(m).exp_()
        total = p.sum(2, keepdim=True)
        o[b:e, hs] = (torch.matmul(p, v) / total).transpose(0, 1).to(o.dtype)
        lse[hs, b:e] = (m + total.log())[..., 0]
    return [o, lse]


def _plain_att_bwd(s):
    c, scale = s["case"], s["case"]["d"] ** -0.5
    dq = torch.zeros(c["T"], c["heads"], c["d"], device=DEV)
    dk, dv = (torch.zeros(c["T"], c["kv"], c["d"], device=DEV) for _ in range(2))
    for b, e, ks, hs in _pieces(s):
        m = ks.stop - ks.start
        n = (hs.stop - hs.start) // m
        q, do, o = (_heads(s[x], b, e, hs) for x in ("q", "do", "o"))
        k, v = _heads(s["k"], b, e, ks, n), _heads(s["v"], b, e, ks, n)
        p = torch.matmul(q, k.transpose(1, 2).contiguous()).mul_(scale)
        p.sub_(s["lse"][hs, b:e, None]).exp_()
        i = torch.arange(e - b, device=DEV)
        p.masked_fill_(i[None, :] > i[:, None], 0.0)
        shared = lambda t: t.view(m, n, e - b, c["d"]).sum(1).transpose(0, 1)     # noqa: E731
        dv[b:e, ks] += shared(torch.matmul(p.transpose(1, 2).contiguous(), do))
        ds = torch.matmul(do, v.transpose(1, 2).contiguous())
        ds.sub_((do * o).sum(2, keepdim=True)).mul_(p)
        del p
        dq[b:e, hs] = torch.matmul(ds, k).mul_(scale).transpose(0, 1)
        dk[b:e, ks] += shared(torch.matmul(ds.transpose(1, 2).contiguous(), q).mul_(scale))
    return [t.to(s["q"].dtype) for t in (dq, dk, dv)]


# ------------------------------------------------------------------ work and the definition
def work(case):
    c, e = case, BYTES[case["dtype"]]
    T, d = c["T"], c["d"]
    if c["op"] == "emb_fwd":
        # at most every row of the embedding is read once
        return dict(bytes=min(T, c["V"]) * d * BYTES[c["wdtype"]] + T * d * e + 4 * T, flops=T * d)
    if c["op"] == "emb_bwd":
        rows = 2 * min(T, c["V"]) if c["accumulate"] else c["V"]
        return dict(bytes=T * d * e + rows * d * 4 + 4 * T, flops=T * d)
    if c["op"] == "rotate":
        return dict(bytes=2 * T * c["heads"] * d * e + 4 * T, flops=3 * T * c["heads"] * c["rot"])
    off = _offsets(c)
    pairs = sum((b - a) * (b - a + 1) // 2 for a, b in zip(off, off[1:])) * c["heads"]
    rows = T * d * e * (c["heads"] + c["kv"])          # q and o, or k and v, twice
    if c["op"] == "att_fwd":
        return dict(bytes=2 * rows + 4 * T * c["heads"], flops=4 * d * pairs)
    return dict(bytes=4 * rows + 4 * T * c["heads"], flops=10 * d * pairs)


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"].startswith("emb"):
        live = torch.ones(c["T"], device=DEV).bool() if s["live"] is None else s["live"].bool()
        if c["op"] == "emb_fwd":
            y = torch.zeros(c["T"], c["d"], dtype=torch.float64, device=DEV)
            y[live] = s["weight"][s["ids"].long()[live]].double() * c["scale"]
            return [y]
        # rows in the order of their ids; a row's sum is a difference of running totals of its run
        order = torch.argsort(s["ids"].long(), stable=True)
        order = order[live[order]]
        dw = s["dweight"].double() if c["accumulate"] else torch.zeros(c["V"], c["d"], dtype=torch.float64, device=DEV)
        ids, n = torch.unique_consecutive(s["ids"].long()[order], return_counts=True)
        at = 0
        for group in torch.split(torch.stack([ids, n], 1).cpu(), 1 << 12):
            rows = int(group[:, 1].sum())
            part = torch.zeros(len(group), c["d"], dtype=torch.float64, device=DEV)
            which = torch.repeat_interleave(torch.arange(len(group)), group[:, 1]).to(DEV)
            part.index_add_(0, which, s["dy"][order[at:at + rows]].double())
            dw[group[:, 0].to(DEV)] += part * c["scale"]
            at += rows
        return [dw]
    if c["op"] == "rotate":
        x, r = s["x"].double(), c["rot"]
        # as complex numbers times a unit one
        pairs = x[..., :r].unflatten(2, (r // 2, 2)) if c["interleaved"] else \
            x[..., :r].unflatten(2, (2, r // 2)).transpose(2, 3)
        i = torch.arange(r // 2, dtype=torch.float64, device=DEV)
        a = s["position"].double()[:, None, None] / c["base"] ** (2 * i / max(r, 1))
        z = torch.view_as_complex(pairs.contiguous()) * torch.polar(torch.ones_like(a), -a if c["inverse"] else a)
        z = torch.view_as_real(z)
        z = z.flatten(2) if c["interleaved"] else z.transpose(2, 3).flatten(2)
        return [torch.cat([z, x[..., r:]], 2)]
    T, h, kv, d = c["T"], c["heads"], c["kv"], c["d"]
    new = lambda *n: torch.zeros(*n, dtype=torch.float64, device=DEV)              # noqa: E731
    o, lse, dq, dk, dv = new(T, h, d), new(h, T), new(T, h, d), new(T, kv, d), new(T, kv, d)
    q, k, v = s["q"], s["k"], s["v"]
    for b, e in zip(s["off"], s["off"][1:]):
        for j in range(h):
            # blocks of rows, each with all the keys it sees
            g = j * kv // h
            for r0 in range(b, e, 4096):
                r1 = min(e, r0 + 4096)
                kk, vv = k[b:r1, g].double(), v[b:r1, g].double()
                w = q[r0:r1, j].double() @ kk.T / math.sqrt(d)
                seen = torch.arange(b, r1, device=DEV)[None, :] <= torch.arange(r0, r1, device=DEV)[:, None]
                w = torch.where(seen, w, -math.inf)
                z = torch.logsumexp(w, 1, keepdim=True)
                w = torch.exp(w - z)
                if c["op"] == "att_fwd":
                    o[r0:r1, j], lse[j, r0:r1] = w @ vv, z[:, 0]
                    continue
                g_o = s["do"][r0:r1, j].double()
                dv[b:r1, g] += w.T @ g_o
                dw = g_o @ vv.T
                dw = w * (dw - (w * dw).sum(1, keepdim=True)) / math.sqrt(d)
                dq[r0:r1, j] = dw @ kk
                dk[b:r1, g] += dw.T @ q[r0:r1, j].double()
    return [o, lse] if c["op"] == "att_fwd" else [dq, dk, dv]
