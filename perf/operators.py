"""The operators around the fused policy loss that are timed: the final norm and the update.

Four operators, each as a trainer meets it:

  norm_fwd   the final layer or RMS norm of a packed micro-batch, which makes the hidden
             states H that the policy loss reads (``TokenNorm.forward``);
  norm_bwd   its backward: dx and the weight's and bias's gradients out of the loss's dH,
             which is zero on observation tokens (``TokenNorm.backward``);
  orth       a gradient or momentum matrix (or a stack of them) made near-orthogonal by five
             Newton-Schulz steps (``Orthogonalize``);
  muon       one optimiser step: momentum, the same products, the weight's update
             (``MuonStep``).

``run`` computes either the plain form in 32 bits with elementary torch operations, or calls
the framework (``own``); ``exact`` computes the definitions in 64 bits.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda"
EPS_NORM = 1e-5
EPS_NS = 1e-7
STEPS = 5
A_NS, B_NS, C_NS = 3.4445, -4.7750, 2.0315      # the quintic of the published optimiser
LR, MU, WD = 0.02, 0.95, 0.1
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BYTES = {"bf16": 2, "f32": 4}


# ------------------------------------------------------------------ the cases
def listed():
    fwd = dict(op="norm_fwd", kind="layer", dtype="bf16", wdtype="f32", masked=False, pitch=0)
    bwd = dict(op="norm_bwd", kind="layer", dtype="bf16", wdtype="f32", dy="f32", masked=True,
               pitch=0)
    orth = dict(op="orth", batch=1, dtype="f32", out="bf16", pitch=0)
    muon = dict(op="muon", batch=1, dtype="f32", out="f32", pitch=0)
    return [
        # one token of a toy model (a decode step's final norm): launch and latency
        dict(fwd, name="norm fwd one token", T=1, d=256, dtype="f32"),
        # an unpadded odd width, rows cut out of a wider buffer, ragged token count
        dict(fwd, name="norm fwd odd width", T=3823, d=1001, wdtype="bf16", pitch=24),
        # the 32B-shaped micro-batch: RMS norm of the action tokens of 64k packed tokens
        dict(fwd, name="norm fwd 64k rms masked", T=65536, d=5120, kind="rms", masked=True,
             wdtype="bf16"),
        # a debugging run's whole micro-batch in fp32
        dict(bwd, name="norm bwd toy", T=1519, d=256, dtype="f32", masked=False),
        # the 7B-shaped micro-batch as the loss leaves it: fp32 dH, a third of the rows live
        dict(bwd, name="norm bwd 32k masked", T=32768, d=3584),
        # a norm inside the decoder: every row live, the gradient in bf16
        dict(bwd, name="norm bwd 64k rms dense", T=65536, d=4096, kind="rms", dy="bf16",
             masked=False, wdtype="bf16"),
        # a small projection or adapter: fifteen small products, latency
        dict(orth, name="orth small", m=128, n=512, dtype="bf16"),
        # no side a multiple of a tile, more rows than columns, rows of a wider buffer
        dict(orth, name="orth odd tall", m=2731, n=1001, pitch=7),
        # a stack of per-layer projections of one shape, result in fp32
        dict(orth, name="orth stack f32", m=1024, n=1024, batch=8, out="f32"),
        # a hidden projection of the 32B-shaped model
        dict(orth, name="orth 5120 square", m=5120, n=5120),
        # a toy model's fp32 weight
        dict(muon, name="muon toy", m=256, n=256),
        # an expanding projection of the 7B-shaped model in bf16, fp32 momentum and gradient
        dict(muon, name="muon 4d x d", m=14336, n=3584, out="bf16"),
    ]


def _log(rng, lo, hi):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return v + 1 if v == 3072 else v


def _size(rng, lo, hi):
    """Log-uniform; half of them odd or otherwise ragged, the others multiples of 64."""
    v = _log(rng, lo, hi)
    return v // 64 * 64 if rng.random() < 0.5 and v >= 64 and v // 64 != 48 else v


def draw(rng):
    op = rng.choice(["norm_fwd", "norm_bwd", "orth", "muon"])
    if op.startswith("norm"):
        T, d = _log(rng, 1, 131072), _size(rng, 64, 8192)
        T = max(1, min(T, 65536 * 5120 // d))
        c = dict(op=op, kind=rng.choice(["layer", "rms"]), dtype=rng.choice(["bf16", "bf16", "f32"]),
                 wdtype=rng.choice(["bf16", "f32"]), masked=rng.random() < 0.5,
                 pitch=rng.choice([0, 0, 64, 5]), T=T, d=d)
        if op == "norm_bwd":
            c["dy"] = rng.choice(["f32", "f32", "bf16"])
        return c
    r = _size(rng, 16, 4096)                 # the shorter side
    c = min(_size(rng, r, 8 * r), 14336)
    batch = rng.choice([1, 1, 1, 2, 6])
    cost = lambda: batch * r * r * (3 * c + r)                                    # noqa: E731
    most = 3584 * 3584 * (3 * 14336 + 3584)
    while batch > 1 and cost() > most:
        batch //= 2
    while cost() > most:
        c = max(r, c * 3 // 4 - 1)
    m, n = (r, c) if rng.random() < 0.5 else (c, r)
    return dict(op=op, m=m, n=n, batch=batch, dtype=rng.choice(["bf16", "f32"]),
                out=rng.choice(["bf16", "bf16", "f32"]), pitch=rng.choice([0, 0, 0, 8, 3]))


# ------------------------------------------------------------------ inputs
def _turns(T, seed):
    """uint8 action mask of a packed stream: turns of 64..512 observation and 32..256 action tokens."""
    rng = np.random.default_rng([seed, 7])
    n = T // 96 + 2
    at = np.cumsum(np.stack([rng.integers(64, 513, n), rng.integers(32, 257, n)], 1).reshape(-1))
    at -= rng.integers(0, 400)               # a micro-batch starts anywhere in a trajectory
    m = (np.searchsorted(at, np.arange(T), side="right") % 2).astype(np.uint8)
    m[T - 1] = 1                             # short ones too have a token that counts
    return m


def _rows(t, pitch):
    """The same rows in a buffer that is `pitch` elements wider."""
    if not pitch:
        return t
    wide = torch.zeros(*t.shape[:-1], t.shape[-1] + pitch, dtype=t.dtype, device=t.device)
    wide[..., : t.shape[-1]] = t
    return wide[..., : t.shape[-1]]


def _matrix(g, batch, m, n):
    """Gradients of a projection: a few strong directions over noise."""
    k = min(12, m, n)
    u = torch.randn(batch, m, k, generator=g, device=DEV) * 0.6 ** torch.arange(k, device=DEV)
    v = torch.randn(batch, k, n, generator=g, device=DEV)
    return (torch.baddbmm(torch.randn(batch, m, n, generator=g, device=DEV), u, v, beta=0.3)).mul_(1e-3)


def prepare(case, seed):
    c, g = case, torch.Generator(device=DEV).manual_seed(seed)
    s = dict(case=c)
    if c["op"].startswith("norm"):
        T, d, dt = c["T"], c["d"], DTYPES[c["dtype"]]
        randn = lambda *n: torch.randn(*n, generator=g, device=DEV)               # noqa: E731
        # residual streams: a few wide channels, a small offset, rows of different scale
        x = randn(T, d)
        x *= torch.exp(0.5 * randn(T, 1))
        x *= torch.where(torch.rand(d, generator=g, device=DEV) < 0.01, 12.0, 1.0)
        x += 0.2
        s["x"] = _rows(x.to(dt), c["pitch"])
        s["weight"] = (1 + 0.2 * randn(d)).to(DTYPES[c["wdtype"]])
        s["bias"] = (0.2 * randn(d)).to(DTYPES[c["wdtype"]]) if c["kind"] == "layer" else None
        s["mask"] = torch.from_numpy(_turns(T, seed)).to(DEV) if c["masked"] else None
        if c["op"] == "norm_bwd":
            dy = randn(T, d) * 1e-2
            if c["masked"]:
                dy *= s["mask"][:, None]
            s["dy"] = _rows(dy.to(DTYPES[c["dy"]]), c["pitch"])
            _, s["mean"], s["rstd"] = _plain_norm_fwd(s)     # what the forward left
    else:
        b, m, n = c["batch"], c["m"], c["n"]
        s["grad"] = _rows(_matrix(g, b, m, n).to(DTYPES[c["dtype"]]), c["pitch"])
        if c["op"] == "muon":
            s["momentum"] = _matrix(g, b, m, n).mul_(1 / (1 - MU))
            s["param"] = torch.randn(b, m, n, generator=g, device=DEV).mul_(0.02).to(DTYPES[c["out"]])
    if own:
        # the handle a program keeps: workspace and outputs of one shape
        import paper_2510_04206_amd as P
        if c["op"].startswith("norm"):
            s["op"] = P.TokenNorm(c["T"], c["d"], dt, kind=c["kind"], eps=EPS_NORM,
                                  grads=c["op"] == "norm_bwd", device=DEV)
            if c["op"] == "norm_bwd":
                if s["mean"] is not None:
                    s["op"].mean.copy_(s["mean"])
                s["op"].rstd.copy_(s["rstd"])
        elif c["op"] == "orth":
            s["op"] = P.Orthogonalize(c["m"], c["n"], out_dtype=DTYPES[c["out"]], batch=c["batch"],
                                      steps=STEPS, coeffs=(A_NS, B_NS, C_NS), eps=EPS_NS, device=DEV)
        else:
            s["op"] = P.MuonStep(c["m"], c["n"], param_dtype=DTYPES[c["out"]], batch=c["batch"],
                                 momentum=MU, nesterov=True, weight_decay=WD, steps=STEPS,
                                 coeffs=(A_NS, B_NS, C_NS), eps=EPS_NS, device=DEV)
    return s


# ------------------------------------------------------------------ one pass
def run(s):
    if own:
        return _run_own(s)
    return {"norm_fwd": _plain_norm_fwd, "norm_bwd": _plain_norm_bwd, "orth": _plain_orth,
            "muon": _plain_muon}[s["case"]["op"]](s)


def _run_own(s):
    kind = s["case"]["op"]
    if kind == "norm_fwd":
        return list(s["op"].forward(s["x"], s["weight"], s["bias"], s["mask"]))
    if kind == "norm_bwd":
        return list(s["op"].backward(s["x"], s["weight"], s["dy"], s["mask"]))
    if kind == "orth":
        return [s["op"](s["grad"])]
    s["op"](s["param"], s["grad"], s["momentum"], LR)
    return [s["param"], s["momentum"]]


def _live(s, t):
    """t on action tokens, 0 elsewhere."""
    if s["mask"] is None:
        return t
    m = s["mask"].bool()
    return torch.where(m[:, None] if t.dim() == 2 else m, t, torch.zeros((), device=DEV))


def _plain_norm_fwd(s):
    x = s["x"].float()
    if s["case"]["kind"] == "layer":
        mean = x.mean(1)
        xc = x - mean[:, None]
    else:
        mean, xc = None, x
    rstd = torch.rsqrt((xc * xc).mean(1) + EPS_NORM)
    y = xc * rstd[:, None] * s["weight"].float()
    if s["bias"] is not None:
        y = y + s["bias"].float()
    return [_live(s, y).to(s["x"].dtype), None if mean is None else _live(s, mean), _live(s, rstd)]


def _plain_norm_bwd(s):
    layer = s["case"]["kind"] == "layer"
    x = s["x"].float()
    xh = (x - s["mean"][:, None] if layer else x) * s["rstd"][:, None]
    dy = _live(s, s["dy"].float())
    g = dy * s["weight"].float()
    c2 = (g * xh).mean(1, keepdim=True)
    dx = g - xh * c2
    if layer:
        dx = dx - g.mean(1, keepdim=True)
    dx = _live(s, dx * s["rstd"][:, None]).to(s["x"].dtype)
    return [dx, (dy * xh).sum(0), dy.sum(0) if layer else None]


def _plain_ns(u):
    """Newton-Schulz steps on a stack of fp32 matrices, on the side with fewer rows."""
    tall = u.shape[1] > u.shape[2]
    x = u.transpose(1, 2).contiguous() if tall else u
    x = x / ((x * x).sum((1, 2), keepdim=True).sqrt() + EPS_NS)
    for _ in range(STEPS):
        a = torch.bmm(x, x.transpose(1, 2).contiguous())
        b = B_NS * a + C_NS * torch.bmm(a, a)
        x = A_NS * x + torch.bmm(b, x)
    return x.transpose(1, 2).contiguous() if tall else x


def _plain_orth(s):
    return [_plain_ns(s["grad"].float()).to(DTYPES[s["case"]["out"]])]


def _plain_muon(s):
    c, grad = s["case"], s["grad"].float()
    s["momentum"].mul_(MU).add_(grad)
    o = _plain_ns(grad + MU * s["momentum"])
    w = (1 - LR * WD) * s["param"].float() - LR * math.sqrt(max(1.0, c["m"] / c["n"])) * o
    s["param"].copy_(w)
    return [s["param"], s["momentum"]]


# ------------------------------------------------------------------ work and the definition
def work(case):
    c = case
    if c["op"].startswith("norm"):
        T, d, e = c["T"], c["d"], BYTES[c["dtype"]]
        live = T / 3 if c["masked"] else T       # a turn is two thirds observation on average
        par = d * BYTES[c["wdtype"]] * (2 if c["kind"] == "layer" else 1)
        if c["op"] == "norm_fwd":
            return dict(bytes=live * d * e + T * d * e + par + 8 * T + (T if c["masked"] else 0),
                        flops=8 * live * d)
        return dict(bytes=live * d * (e + BYTES[c["dy"]]) + T * d * e + par + 8 * live +
                    4 * d * (2 if c["kind"] == "layer" else 1) + (T if c["masked"] else 0),
                    flops=14 * live * d)
    b, m, n = c["batch"], c["m"], c["n"]
    r, k = min(m, n), max(m, n)
    by = BYTES[c["dtype"]] + BYTES[c["out"]] + (8 + BYTES[c["out"]] if c["op"] == "muon" else 0)
    # the two symmetric products need half of their entries
    return dict(bytes=b * m * n * by, flops=b * STEPS * (3.0 * r * r * k + 1.0 * r * r * r))


def _polar_64(u):
    """The same polynomial on the longer side's vectors: X <- X (a + b K + c K K), K = X^T X (or its transpose)."""
    out = []
    for x in u.double():
        wide = x.shape[0] <= x.shape[1]
        x = x / (torch.linalg.matrix_norm(x) + EPS_NS)
        eye = torch.eye(min(x.shape), dtype=torch.float64, device=x.device)
        for _ in range(STEPS):
            k = x @ x.mT if wide else x.mT @ x
            p = A_NS * eye + k @ (B_NS * eye + C_NS * k)
            x = p @ x if wide else x @ p
        out.append(x)
    return torch.stack(out)


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"].startswith("norm"):
        x, w = s["x"].double(), s["weight"].double()
        live = torch.ones(c["T"], device=DEV).bool() if s["mask"] is None else s["mask"].bool()
        x = torch.where(live[:, None], x, 0.0)
        mean = x.sum(1) / c["d"] if c["kind"] == "layer" else torch.zeros(c["T"], device=DEV).double()
        var = x.square().sum(1) / c["d"] - mean.square()
        rstd = torch.where(live, (var + EPS_NORM) ** -0.5, 0.0)
        xh = (x - mean[:, None]) * rstd[:, None]
        if c["op"] == "norm_fwd":
            y = xh * w + (s["bias"].double() if s["bias"] is not None else 0.0)
            return [torch.where(live[:, None], y, 0.0), mean if c["kind"] == "layer" else None, rstd]
        dy = torch.where(live[:, None], s["dy"].double(), 0.0)
        g = dy * w
        # the gradient's component along the directions that the norm removes, taken out
        along = (g * xh).sum(1, keepdim=True) / c["d"] * xh
        if c["kind"] == "layer":
            along += g.sum(1, keepdim=True) / c["d"]
        dx = (g - along) * rstd[:, None]
        return [dx, (dy * xh).sum(0), dy.sum(0) if c["kind"] == "layer" else None]
    grad = s["grad"].double()
    if c["op"] == "orth":
        return [_polar_64(grad)]
    mom = MU * s["momentum"].double() + grad
    o = _polar_64(grad + MU * mom)
    w = s["param"].double()
    return [w - LR * WD * w - LR * max(1.0, c["m"] / c["n"]) ** 0.5 * o, mom]
