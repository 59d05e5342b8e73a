"""One decoder block over packed trajectories, from token ids to the policy loss and back.

    ids --embed--> x --norm, q k v (torch)--> rotate, attention --project (torch), + x--> h
      --final norm--> H --LM head, policy loss--> L

over one packed micro-batch: trajectories end to end, each attending to itself alone, positions
counted from its first token, padding behind the last one in no sequence.  The head is the embedding:
its gradient is the loss's dW with the embedding's rows added in place.

    forward     TokenEmbedding, TokenNorm, TokenRotation, PackedAttention, TokenNorm, PolicyLoss
    backward    the same in turn; the projections' gradients are torch products

Run it on a GPU with ``python examples/trunk_step.py [--steps N]``.
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2510_04206_amd as P                                                # noqa: E402
from workloads import gen                                                       # noqa: E402


def packing(traj_id):
    """Offsets of the trajectories in a packed stream, and each token's position in its own (host arrays).
    Padding (id -1) lies behind the last one."""
    t = np.asarray(traj_id)
    n = int((t >= 0).sum())
    start = np.concatenate([[0], np.flatnonzero(np.diff(t[:n])) + 1, [n]]).astype(np.int32)
    position = np.zeros(len(t), np.int32)
    position[:n] = np.arange(n) - np.repeat(start[:-1], np.diff(start))
    return start, position


class Block:
    """Parameters and handles of one micro-batch shape."""

    def __init__(self, T, V, d, n_head, n_kv, n_act, dtype=torch.bfloat16, seed=0, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        self.T, self.d, self.n_head, self.n_kv, self.dh, self.dtype = T, d, n_head, n_kv, d // n_head, dtype
        new = lambda *n: torch.randn(*n, generator=g, device=device)             # noqa: E731
        self.embedding = 0.02 * new(V, d)
        self.wqkv = new((n_head + 2 * n_kv) * self.dh, d) / d ** 0.5
        self.wo = new(d, d) / d ** 0.5
        self.gamma1, self.gamma2 = torch.ones(d, device=device), torch.ones(d, device=device)
        self.loss = P.PolicyLoss(T, d, V, dtype, max_act=n_act, device=device)
        self.embed = P.TokenEmbedding(T, V, d, dtype, scale=d ** 0.5, dweight=self.loss.dW, device=device)
        self.norm1, self.norm2 = (P.TokenNorm(T, d, dtype, kind="rms", device=device) for _ in range(2))
        self.rotate = P.TokenRotation(T, n_head + n_kv, self.dh, dtype, output=False, device=device)
        self.attend = P.PackedAttention(T, n_head, n_kv, self.dh, dtype, device=device)

    def forward(self, ids, live, start, position):
        """Everything up to H; what the backward needs stays on the handle and in `self.saved`."""
        W = self.embedding.to(self.dtype)
        x = self.embed.forward(W, ids, live)
        y = self.norm1.forward(x, self.gamma1, None, live)[0]
        qkv = (y.float() @ self.wqkv.t()).to(self.dtype).view(self.T, self.n_head + 2 * self.n_kv, self.dh)
        turned = qkv[:, : self.n_head + self.n_kv]
        self.rotate(turned, position, out=turned)
        q, k, v = qkv.split((self.n_head, self.n_kv, self.n_kv), 1)
        o = self.attend.forward(q, k, v, start)[0].view(self.T, self.d)
        h = (x.float() + o.float() @ self.wo.t()).to(self.dtype)
        H = self.norm2.forward(h, self.gamma2, None, live)[0]
        self.saved = (W, x, y, q, k, v, o, h, H)
        return H, W

    def backward(self, ids, live, start, position, mask, adv, old_logp):
        """Gradients by name; the embedding's is the tied [V, d] one."""
        W, x, y, q, k, v, o, h, H = self.saved
        dH, dW = self.loss.backward(H, W, ids, mask, adv, old_logp)
        dh, dgamma2, _ = self.norm2.backward(h, self.gamma2, dH, live)
        dh = dh.float()
        do = (dh @ self.wo).to(self.dtype).view(self.T, self.n_head, self.dh)
        dwo = dh.t() @ o.float()
        self.attend.backward(q, k, v, start, do)
        dqkv = self.attend.dqkv
        turned = dqkv[:, : self.n_head + self.n_kv]
        self.rotate(turned, position, inverse=True, out=turned)
        dqkv = dqkv.view(self.T, -1).float()
        dy, dwqkv = dqkv @ self.wqkv, dqkv.t() @ y.float()
        dx, dgamma1, _ = self.norm1.backward(x, self.gamma1, dy, live)
        self.embed.backward(ids, dx.float() + dh, live, accumulate=True)
        return dict(embedding=dW, wqkv=dwqkv, wo=dwo, gamma1=dgamma1, gamma2=dgamma2)

    def step(self, ids, live, start, position, mask, adv, old_logp, lr):
        H, W = self.forward(ids, live, start, position)
        loss = self.loss.forward(H, W, ids, mask, adv, old_logp)[0].clone()
        for name, g in self.backward(ids, live, start, position, mask, adv, old_logp).items():
            getattr(self, name).sub_(g, alpha=lr)
        return loss


def inputs(w, pad: int = 0):
    """Device arrays of a workload's micro-batch, `pad` tokens of padding behind it."""
    to = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()              # noqa: E731
    more = lambda a, v: np.concatenate([a, np.full(pad, v, a.dtype)])            # noqa: E731
    traj = more(w.traj_id, -1)
    start, position = packing(traj)
    # (ids of observation tokens are embedded too: the workload draws action tokens' only)
    ids = np.where(w.mask, w.token_id, np.arange(w.T) * 7919 % w.V).astype(np.int32)
    return dict(ids=to(more(ids, 0)), live=to((traj >= 0).astype(np.uint8)), start=to(start), position=to(position)), \
        to(more(w.mask, 0))


def run(steps: int = 6, V: int = 1000, d: int = 128, seed: int = 1, lr: float = 0.02):
    """The loss of each step on one small synthetic micro-batch."""
    w = gen.make(gen.small_spec(V=V, d=d, dtype="bf16", name="trunk"), seed=seed)
    at, mask = inputs(w, pad=5)
    T = w.T + 5
    g = torch.Generator(device="cuda").manual_seed(seed)
    adv = torch.randn(T, generator=g, device="cuda")
    block = Block(T, V, d, 4, 2, w.n_act, seed=seed)
    H, W = block.forward(**at)
    old = P.TokenLogprob(T, d, V, torch.bfloat16, max_act=w.n_act)(H, W, at["ids"], mask)[0].clone()
    losses = [float(block.step(**at, mask=mask, adv=adv, old_logp=old, lr=lr)) for _ in range(steps)]
    if P.agrl_get_device_error():
        raise RuntimeError("a kernel found an index out of range")
    return losses


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=6)
    for i, loss in enumerate(run(ap.parse_args().steps)):
        print(f"step {i}: loss {loss:+.5f}", flush=True)


if __name__ == "__main__":
    main()
