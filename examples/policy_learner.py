"""A recurrent policy trained with the policy operators alone: acting by single steps, learning over whole sequences.

The task needs a memory: the first observation shows one of A signs, all others are blank, and the action of the last step is
rewarded if it is that sign.  The policy is one projection to (x, r, i), the gated linear recurrence, and one projection to
the logits.

    acting     marl_linear_step on a table of states, marl_log_prob for the likeliest action
    learning   marl_linear_scan, marl_log_prob, marl_log_prob_grad, marl_linear_scan_grad, marl_muon_step

    python examples/policy_learner.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2205_05248_amd import binding  # noqa: E402

DECAY = 8.0
ENTROPY_BONUS = 0.01


def _bytes(n):
    return torch.empty(max(n, 1), dtype=torch.uint8, device="cuda")


class Policy:
    """Weights, momenta, and the buffers of a batch of B sequences of T steps, all on the device."""

    def __init__(self, B, T, signs, C=64, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.B, self.T, self.A, self.C, self.D = B, T, signs, C, signs + 1
        new = lambda *shape: torch.zeros(*shape, device="cuda")
        self.w_in = (torch.randn(3 * C, self.D, generator=g) * 0.5).cuda()
        self.w_out = (torch.randn(self.A, C, generator=g) * 0.1).cuda()
        self.lam = torch.log(torch.expm1(-torch.log(0.9 + 0.099 * torch.rand(C, generator=g)))).cuda()
        self.m_in, self.m_out = torch.zeros_like(self.w_in), torch.zeros_like(self.w_out)
        self.y, self.logits, self.grad_logits = new(B, T, C), new(B * T, self.A), new(B * T, self.A)
        self.logp, self.entropy, self.log_sum = new(B * T), new(B * T), new(B * T)
        self.grad_proj, self.grad_y, self.grad_lam = new(B, T, 3 * C), new(B, T, C), new(C)
        self.state, self.step_y = new(B, C), new(B, C)
        self.best, self.best_logp = torch.zeros(B, 1, dtype=torch.int32, device="cuda"), new(B, 1)
        self.ws_scan = _bytes(binding.marl_linear_scan_workspace_bytes("fp32", B, T, C))
        self.ws_logp = _bytes(binding.marl_log_prob_workspace_bytes(B * T, self.A, 1))
        self.ws_in = _bytes(binding.marl_muon_workspace_bytes("fp32", 1, 3 * C, self.D))
        self.ws_out = _bytes(binding.marl_muon_workspace_bytes("fp32", 1, self.A, C))

    def _gates(self, proj):
        return tuple(proj[..., k * self.C:(k + 1) * self.C] for k in range(3))

    def act(self, obs, first, noise=None):
        """One action [B] for observations [B,D]; first: the sequences begin here.  noise [B,A] is added to the logits (Gumbel noise samples)."""
        reset = torch.full((self.B,), int(first), dtype=torch.uint8, device="cuda")
        binding.marl_linear_step(*self._gates(obs @ self.w_in.t()), self.lam, DECAY, None, reset, self.state, self.state, self.step_y)
        logits = self.step_y @ self.w_out.t()
        if noise is not None:
            logits += noise
        binding.marl_log_prob(logits, None, None, 1.0, None, None, None, self.best, self.best_logp, self.ws_logp)
        return self.best[:, 0].clone()

    def gradient(self, obs, action, advantage):
        """Of -mean(advantage log p(action) + bonus entropy) over obs [B,T,D], action [B,T] i32, advantage [B,T]."""
        n = self.B * self.T
        token, reset = action.reshape(-1), torch.zeros(self.B, self.T, dtype=torch.uint8, device="cuda")
        reset[:, 0] = 1
        x, r, i = self._gates(obs @ self.w_in.t())
        binding.marl_linear_scan(x, r, i, self.lam, DECAY, reset, None, None, self.y, None, self.ws_scan)
        torch.matmul(self.y.view(n, self.C), self.w_out.t(), out=self.logits)
        binding.marl_log_prob(self.logits, token, None, 1.0, self.logp, self.entropy, self.log_sum, workspace=self.ws_logp)
        binding.marl_log_prob_grad(self.logits, token, None, 1.0, self.log_sum, self.entropy, advantage.reshape(-1) * (-1.0 / n),
                                   torch.full((n,), -ENTROPY_BONUS / n, device="cuda"), self.grad_logits)
        torch.matmul(self.grad_logits, self.w_out, out=self.grad_y.view(n, self.C))
        binding.marl_linear_scan_grad(x, r, i, self.lam, DECAY, reset, None, self.grad_y, None, self.ws_scan, *self._gates(self.grad_proj),
                                      self.grad_lam)
        grad_in = self.grad_proj.view(n, 3 * self.C).t() @ obs.reshape(n, self.D)
        return grad_in, self.grad_logits.t() @ self.y.view(n, self.C), self.grad_lam

    def update(self, grad_in, grad_out, grad_lam, lr=0.05):
        binding.marl_muon_step(self.w_in, grad_in.contiguous(), self.m_in, self.w_in, self.m_in, self.ws_in, lr=lr)
        binding.marl_muon_step(self.w_out, grad_out.contiguous(), self.m_out, self.w_out, self.m_out, self.ws_out, lr=lr)
        self.lam -= lr * grad_lam


def observations(signs, T, A):
    obs = torch.zeros(len(signs), T, A + 1, device="cuda")
    obs[:, 1:, A] = 1.0
    obs[torch.arange(len(signs), device="cuda"), 0, signs] = 1.0
    return obs


def play(policy, generator=None):
    """Signs [B], observations [B,T,D], actions [B,T] of one batch; without a generator the signs go round and the likeliest actions are taken."""
    B, T, A = policy.B, policy.T, policy.A
    signs = torch.arange(B, device="cuda") % A if generator is None else torch.randint(A, (B,), generator=generator, device="cuda")
    obs, actions = observations(signs, T, A), []
    for t in range(T):
        noise = None if generator is None else -torch.log(-torch.log(torch.rand(B, A, generator=generator, device="cuda").clamp(1e-7, 1 - 1e-7)))
        actions.append(policy.act(obs[:, t], t == 0, noise))
    return signs, obs, torch.stack(actions, 1)


def success(policy):
    signs, _, actions = play(policy)
    return (actions[:, -1] == signs).float().mean().item()


def train(iterations=150, B=256, T=12, A=5, seed=0, report=None):
    """A trained policy; report(iteration, share of rewarded sequences) every 25 iterations."""
    policy, g = Policy(B, T, A, seed=seed), torch.Generator(device="cuda").manual_seed(seed)
    for k in range(iterations):
        signs, obs, actions = play(policy, g)
        reward = (actions[:, -1] == signs).float()
        advantage = torch.zeros(B, T, device="cuda")
        advantage[:, -1] = reward - reward.mean()
        policy.update(*policy.gradient(obs, actions, advantage), lr=0.05 * (1 - k / iterations))
        if report and k % 25 == 24:
            report(k + 1, success(policy))
    return policy


if __name__ == "__main__":
    train(report=lambda k, s: print(f"iteration {k}: {s:.3f} of the signs remembered", flush=True))
