"""The policy operators together: gradient of a whole recurrent policy against 64-bit autograd, and that it learns.

Tolerance of the gradient: that of the parts, 250 * 2^-21 of the largest entry (the recurrence's) for each of the two chains a
gradient has gone through, and the fp32 products' sqrt(K) 2^-24 over K = B T = 84 terms, which is below it.
"""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
pytestmark = pytest.mark.gpu


def test_gradient_of_the_whole_policy():
    import policy_learner as pl
    B, T, A, C = 12, 7, 4, 24
    p = pl.Policy(B, T, A, C, seed=3)
    g = torch.Generator().manual_seed(4)
    obs, action = torch.randn(B, T, A + 1, generator=g), torch.randint(A, (B, T), generator=g).to(torch.int32)
    advantage = torch.randn(B, T, generator=g)
    got = [v.clone() for v in p.gradient(obs.cuda(), action.cuda(), advantage.cuda())]
    torch.cuda.synchronize()
    w_in, w_out, lam = (v.double().cpu().requires_grad_() for v in (p.w_in, p.w_out, p.lam))
    x, r, i = (obs.double() @ w_in.t()).split(C, -1)
    rate = pl.DECAY * torch.log1p(torch.exp(lam))
    h, ys = None, []
    for t in range(T):
        log_a = -rate * torch.sigmoid(r[:, t])
        u = torch.sigmoid(i[:, t]) * x[:, t]
        h = u if t == 0 else torch.exp(log_a) * h + torch.sqrt(1 - torch.exp(2 * log_a)) * u
        ys.append(h)
    logp = torch.log_softmax(torch.stack(ys, 1) @ w_out.t(), -1)
    taken = logp.gather(-1, action.long()[..., None])[..., 0]
    loss = -(advantage.double() * taken + pl.ENTROPY_BONUS * -(logp.exp() * logp).sum(-1)).mean()
    loss.backward()
    for have, want in zip(got, (w_in.grad, w_out.grad, lam.grad)):
        assert (have.double().cpu() - want).abs().max() <= 2 * 250 * 2.0 ** -21 * want.abs().max()


def test_it_learns_to_remember():
    import policy_learner as pl
    assert pl.success(pl.train(iterations=150)) >= 0.9
