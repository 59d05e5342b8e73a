"""The example's steps: the operators together, their gradients against autograd, the loss falls."""
import os
import sys

import numpy as np
import pytest
import torch

from helpers import log

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_loss_falls(kind):
    """The clipped surrogate starts at ratio 1 and every step follows its gradient; after eight the
    loss has fallen, by more than the first step's rounding (bf16: 2^-8 of the advantages' size 1)."""
    import policy_step
    log(f"example {kind}")
    losses = policy_step.run(steps=8, kind=kind)
    log("  " + " ".join(f"{v:+.4f}" for v in losses))
    assert all(np.isfinite(losses))
    assert losses[-1] < losses[0] - 2 ** -8


@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_gradients_of_the_chain(kind):
    """dproj and dgamma of one step against autograd in 64 bits through the same chain.  bf16
    activations and logit gradients (2^-9 each, three of them in a row): 1e-2."""
    import policy_step
    import paper_2510_04206_amd as P
    from workloads import gen
    log(f"example gradients {kind}")
    w = gen.make(gen.small_spec(V=500, d=64, dtype="bf16", name="example"), seed=3)
    to = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()              # noqa: E731
    mask, ids, x = to(w.mask), to(w.token_id), w.H.cuda()
    adv = to(np.random.default_rng(0).standard_normal(w.T).astype(np.float32))
    top = policy_step.Top(w, kind=kind, seed=3)
    old = top.behaviour(x, ids, mask)
    h, H, W = top.hidden(x, mask)
    top.loss.forward(H, W, ids, mask, adv, old)
    dH, _ = top.loss.backward(H, W, ids, mask, adv, old)
    dh, dgamma, _ = top.norm.backward(h, top.gamma, dH, mask)
    dproj = (dh.float().t() @ x.float()).double().cpu()
    m = mask.bool().cpu()
    proj = top.proj.double().cpu().requires_grad_()
    gamma = top.gamma.double().cpu().requires_grad_()
    hid = x.double().cpu()[m] @ proj.t()
    if kind == "layer":
        hid = hid - hid.mean(1, keepdim=True)
    n = hid / (hid.square().mean(1, keepdim=True) + 1e-5).sqrt() * gamma
    logp = torch.log_softmax(n @ W.double().cpu().t(), 1).gather(1, ids.cpu().long()[m][:, None])[:, 0]
    # (bf16 log-probs of the same model: all ratios within the clip bounds)
    loss = -((logp - old.double().cpu()[m]).exp() * adv.double().cpu()[m]).mean()
    loss.backward()
    for got, want in ((dproj, proj.grad), (dgamma.double().cpu(), gamma.grad)):
        e = float((got - want).norm() / want.norm())
        log(f"  off by {e:.1e}")
        assert e <= 1e-2
    assert P.agrl_get_device_error() == 0
