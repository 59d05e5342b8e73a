"""Training steps of the top of a model with every operator of the library in its place.

The top is one hidden projection, the final norm and the LM head:

    x [T, d] --project--> h --norm--> H --LM head, policy loss--> L

over one packed micro-batch of agent trajectories: observation tokens are masked, so the norm
skips their rows and the loss never reads them.  A step runs

    advantages      task_adv_norm              once per batch of trajectories
    forward         h = x P^T (torch), TokenNorm.forward, PolicyLoss.forward
    backward        PolicyLoss.backward (dH, dW), TokenNorm.backward (dh and the weight's
                    gradient), dP = dh^T x (torch)
    update          MuonStep for the projection, plain gradient steps for the norm's weight
                    and the head

The behaviour policy is the model before the first step, its log-probabilities recomputed with
TokenLogprob.  Run it on a GPU with ``python examples/policy_step.py [--steps N]``.
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


class Top:
    """Parameters, optimiser state and the handles of one micro-batch shape."""

    def __init__(self, w, kind: str = "rms", dtype=torch.bfloat16, seed: int = 0, lr: float = 0.02,
                 head_lr: float = 1.0, norm_lr: float = 0.1, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        d = w.d
        self.dtype, self.lr, self.head_lr, self.norm_lr = dtype, lr, head_lr, norm_lr
        self.proj = torch.randn(d, d, generator=g, device=device) / d ** 0.5
        self.momentum = torch.zeros_like(self.proj)
        self.gamma = torch.ones(d, device=device)
        self.head = w.W.float().to(device)
        self.norm = P.TokenNorm(w.T, d, dtype, kind=kind, bias_grad=False, device=device)
        self.logprob = P.TokenLogprob(w.T, d, w.V, dtype, max_act=w.n_act, device=device)
        self.loss = P.PolicyLoss(w.T, d, w.V, dtype, max_act=w.n_act, device=device)
        self.muon = P.MuonStep(d, d, param_dtype=torch.float32, device=device)

    def hidden(self, x, mask):
        """h and H = norm(h); the head in the compute type."""
        h = (x.float() @ self.proj.t()).to(self.dtype)
        return h, self.norm.forward(h, self.gamma, None, mask)[0], self.head.to(self.dtype)

    def behaviour(self, x, ids, mask):
        _, H, W = self.hidden(x, mask)
        return self.logprob(H, W, ids, mask)[0].clone()

    def step(self, x, ids, mask, adv, old_logp) -> torch.Tensor:
        h, H, W = self.hidden(x, mask)
        loss = self.loss.forward(H, W, ids, mask, adv, old_logp)[0].clone()
        dH, dW = self.loss.backward(H, W, ids, mask, adv, old_logp)
        dh, dgamma, _ = self.norm.backward(h, self.gamma, dH, mask)
        dproj = dh.float().t() @ x.float()
        self.muon(self.proj, dproj, self.momentum, self.lr)
        self.gamma.sub_(dgamma, alpha=self.norm_lr)
        self.head.sub_(dW, alpha=self.head_lr)
        return loss


def run(steps: int = 8, V: int = 1000, d: int = 128, kind: str = "rms", seed: int = 1):
    """The loss of each step on one small synthetic micro-batch."""
    w = gen.make(gen.small_spec(V=V, d=d, dtype="bf16", name="example"), seed=seed)
    to = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()              # noqa: E731
    mask, ids, x = to(w.mask), to(w.token_id), w.H.cuda()
    adv = P.task_adv_norm(to(w.g_traj_id), to(w.g_mask), to(w.traj_task), to(w.traj_group),
                          to(w.reward), w.n_task, w.n_group)["adv_tok"][: w.T]
    top = Top(w, kind=kind, seed=seed)
    old = top.behaviour(x, ids, mask)
    losses = [float(top.step(x, ids, mask, adv, old)) for _ in range(steps)]
    if P.agrl_get_device_error():
        raise RuntimeError("a kernel found an index out of range")
    return losses


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=8)
    ap.add_argument("--kind", choices=("rms", "layer"), default="rms")
    a = ap.parse_args()
    for i, loss in enumerate(run(a.steps, kind=a.kind)):
        print(f"step {i}: loss {loss:+.5f}", flush=True)


if __name__ == "__main__":
    main()
