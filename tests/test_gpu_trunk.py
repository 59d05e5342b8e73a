"""Embedding, norm, rotation, attention and loss together as one decoder block: gradients of every parameter
against autograd in 64 bits through the same chain, and the example's steps."""
import os
import sys

import numpy as np
import pytest
import torch

from helpers import log

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_packing():
    import trunk_step
    start, position = trunk_step.packing([4, 4, 4, 0, 7, 7, -1, -1])
    assert start.tolist() == [0, 3, 4, 6] and position.tolist() == [0, 1, 2, 0, 0, 1, 0, 0]


def test_steps_run():
    import trunk_step
    losses = trunk_step.run(steps=3)
    log("  " + " ".join(f"{v:+.4f}" for v in losses))
    assert len(losses) == 3 and all(np.isfinite(losses))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gradients_of_the_chain(dtype):
    """bf16: about ten roundings of activations and gradients in a row, 2^-8 at most and 2^-9.8 as a root mean square
    each, adding up as such: 10^0.5 2^-9.8 = 3.6e-3 of each gradient's norm, and 2e-2 with what softmax and
    norms amplify them by (a factor of 5).  fp32: as many of 2^-24 and sums of up to 2^10 terms: 1e-4."""
    import paper_2510_04206_amd as P
    import trunk_step
    from workloads import gen
    log(f"trunk gradients {dtype}")
    V, d, heads, kv = 500, 64, 4, 2
    w = gen.make(gen.small_spec(V=V, d=d, dtype="bf16", name="trunk"), seed=3)
    at, mask = trunk_step.inputs(w, pad=7)
    T, dh = w.T + 7, d // heads
    adv = torch.randn(T, generator=torch.Generator().manual_seed(0))
    block = trunk_step.Block(T, V, d, heads, kv, w.n_act, dtype=dtype, seed=3)
    H, W = block.forward(**at)
    old = P.TokenLogprob(T, d, V, dtype, max_act=w.n_act)(H, W, at["ids"], mask)[0].clone()
    block.loss.forward(H, W, at["ids"], mask, adv.cuda(), old)
    got = {k: v.double().cpu() for k, v in block.backward(**at, mask=mask, adv=adv.cuda(), old_logp=old).items()}
    assert P.agrl_get_device_error() == 0

    leaf = {k: getattr(block, k).double().cpu().requires_grad_() for k in got}
    n = int(at["start"][-1])
    ids, pos, st = at["ids"].cpu().long()[:n], at["position"].cpu().double()[:n], at["start"].cpu().tolist()
    rms = lambda x, g: x / (x.square().mean(1, keepdim=True) + 1e-5).sqrt() * g    # noqa: E731
    E = leaf["embedding"]
    if dtype == torch.bfloat16:          # (the weight that was used; its gradient passes the rounding)
        E = E + (E.detach().to(dtype).double() - E.detach())
    x = E[ids] * d ** 0.5
    qkv = (rms(x, leaf["gamma1"]) @ leaf["wqkv"].t()).view(n, heads + 2 * kv, dh)
    ang = pos[:, None] * 10000.0 ** (-2.0 * torch.arange(dh // 2).double() / dh)
    c, s = ang.cos()[:, None], ang.sin()[:, None]
    a, b = qkv[:, : heads + kv, : dh // 2], qkv[:, : heads + kv, dh // 2:]
    qk = torch.cat([a * c - b * s, a * s + b * c], 2)
    q, k, v = qk[:, :heads], qk[:, heads:], qkv[:, heads + kv:]
    out = []
    for i, j in zip(st, st[1:]):
        rep = heads // kv
        S = torch.einsum("nhd,mhd->hnm", q[i:j], k[i:j].repeat_interleave(rep, 1)) / dh ** 0.5
        S = S.masked_fill(torch.ones(j - i, j - i).triu(1).bool(), -torch.inf)
        out.append(torch.einsum("hnm,mhd->nhd", S.softmax(2), v[i:j].repeat_interleave(rep, 1)))
    h = x + torch.cat(out).reshape(n, d) @ leaf["wo"].t()
    m = mask.cpu().bool()[:n]
    logp = torch.log_softmax(rms(h, leaf["gamma2"])[m] @ E.t(), 1).gather(1, ids[m][:, None])[:, 0]
    # (the same model's log-probs: every ratio is within the clip bounds, and its gradient that of the log-prob)
    loss = -(logp * (logp.detach() - old.double().cpu()[:n][m]).exp() * adv.double()[:n][m]).mean()
    loss.backward()
    for name, g in got.items():
        want = leaf[name].grad
        e = float((g - want).norm() / want.norm())
        log(f"  {name} off by {e:.1e}")
        assert e <= (2e-2 if dtype == torch.bfloat16 else 1e-4), name
