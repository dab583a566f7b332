"""The memory and what stands behind it used together, as a learner and a server use them, against the 64-bit oracles put together the same way."""
import numpy as np
import pytest
import torch

from oracle import memory_oracle, policy_oracle
from paper_2205_05248_amd import binding
from policy_util import DT, gen, host, randn

pytestmark = pytest.mark.gpu


def new(*shape, dtype=torch.float32):
    return torch.full(shape, float("nan") if dtype.is_floating_point else 7, dtype=dtype, device="cuda")


def room(n):
    return torch.empty(max(n, 1), dtype=torch.uint8, device="cuda")


class Learner:
    """A batch of padded episodes through the memory, a readout, the divergence from a teacher's alternatives, and all the way back."""

    def __init__(self, B, T, Hk, Hv, Dk, Dv, A, K, seed):
        g = gen(seed)
        unit = lambda t: t / t.norm(dim=-1, keepdim=True)
        self.shape, self.A, self.K = (B, T, Hk, Hv, Dk, Dv), A, K
        length = torch.randint(1, T + 1, (B,), generator=g)
        self.filled = (torch.arange(T)[None] < length[:, None]).to(torch.uint8).cuda()
        self.reset = torch.zeros(B, T, dtype=torch.uint8)
        self.reset[:, 0] = 1
        self.reset = self.reset.cuda()
        self.q, self.k = (unit(randn(g, B, T, Hk, Dk)).cuda() for _ in range(2))
        self.v, self.log_decay, self.beta = randn(g, B, T, Hv, Dv).cuda(), (-0.2 * torch.rand(B, T, Hv, generator=g)).cuda(), torch.rand(B, T, Hv, generator=g).cuda()
        self.w = (randn(g, A, Hv * Dv) * 0.2).cuda()
        self.avail = (torch.rand(B * T, A, generator=g) < 0.8).to(torch.uint8).cuda()
        self.avail[:, 0] = 1
        teacher = (randn(g, B * T, A) * 2).cuda()
        self.top_id, self.top_value = new(B * T, K, dtype=torch.int32), new(B * T, K)
        binding.marl_log_prob(teacher, None, self.avail, 1.0, None, None, None, self.top_id, self.top_value,
                              room(binding.marl_log_prob_workspace_bytes(B * T, A, K)))
        self.grad_loss = self.filled.reshape(-1).float() / float(self.filled.sum())
        self.ws = room(binding.marl_delta_scan_workspace_bytes("fp32", B, T, Hk, Hv, Dk, Dv, True))
        self.ws_loss = room(binding.marl_distill_workspace_bytes(B * T, A, K))
        n = B * T
        self.o, self.logits, self.grad_logits, self.grad_o = new(B, T, Hv, Dv), new(n, A), new(n, A), new(B, T, Hv, Dv)
        self.loss, self.log_sum, self.log_rest = new(n), new(n), new(n)
        self.grad = dict(q=new(B, T, Hk, Dk), k=new(B, T, Hk, Dk), v=new(B, T, Hv, Dv), log_decay=new(B, T, Hv), beta=new(B, T, Hv))
        self.grad_w, self.momentum = new(A, Hv * Dv), torch.zeros_like(self.w)
        self.ws_muon = room(binding.marl_muon_workspace_bytes("fp32", 1, A, Hv * Dv))

    def run(self):
        B, T, Hk, Hv, Dk, Dv = self.shape
        memory = (self.q, self.k, self.v, self.log_decay, self.beta, Dk ** -0.5, self.reset, self.filled)
        binding.marl_delta_scan(*memory, None, self.o, None, self.ws, keep=True)
        rows = self.o.view(B * T, Hv * Dv)
        torch.matmul(rows, self.w.t(), out=self.logits)
        student = (self.logits, self.top_id, self.top_value, self.avail, 1.0, True)
        binding.marl_distill(*student, self.loss, self.log_sum, self.log_rest, self.ws_loss)
        binding.marl_distill_grad(*student, self.log_sum, self.log_rest, self.grad_loss, self.grad_logits)
        torch.matmul(self.grad_logits, self.w, out=self.grad_o.view(B * T, Hv * Dv))
        torch.matmul(self.grad_logits.t(), rows, out=self.grad_w)
        g = self.grad
        binding.marl_delta_scan_grad(*memory, self.grad_o, None, self.ws, g["q"], g["k"], g["v"], g["log_decay"], g["beta"])

    def wanted(self):
        B, T, Hk, Hv, Dk, Dv = self.shape
        h = {n: host(getattr(self, n)) for n in ("q", "k", "v", "log_decay", "beta", "reset", "filled", "w", "avail", "top_id", "top_value", "grad_loss")}
        memory = (h["q"], h["k"], h["v"], h["log_decay"], h["beta"], Dk ** -0.5, h["reset"], h["filled"])
        o, _, _ = memory_oracle.delta_scan(*memory, None)
        logits = o.reshape(B * T, Hv * Dv) @ h["w"].T
        loss = memory_oracle.distill(logits, h["top_id"], h["top_value"], h["avail"], 1.0, 1, h["grad_loss"])
        grad_o = (loss["grad"] @ h["w"]).reshape(o.shape)
        grads = memory_oracle.delta_scan_grad(*memory, None, grad_o, None)
        # o is off by 2^-15 of its largest value, a logit by that times the sum of a row of w (and fewer roundings of the product), a probability by twice
        # that part of itself, and as much again comes from grad_o's own product and from the way back
        off = 2.0 ** -15 * (4 * np.abs(o).max() * np.abs(h["w"]).sum(1).max() + 4)
        return loss, loss["grad"].T @ o.reshape(B * T, -1), dict(zip(("q", "k", "v", "log_decay", "beta"), grads)), off


@pytest.mark.parametrize("shape,A,K", [((3, 70, 2, 4, 24, 20), 40, 8), ((4, 9, 1, 2, 16, 16), 11, 3), ((1, 130, 1, 1, 64, 33), 3000, 16)])
def test_loss_and_gradients_of_a_batch(shape, A, K):
    learner = Learner(*shape, A, K, 3)
    learner.run()
    torch.cuda.synchronize()
    loss, grad_w, grads, off = learner.wanted()
    live = host(learner.filled).reshape(-1) != 0
    assert np.abs(host(learner.loss) - loss["loss"])[live].max() <= off * max(1.0, np.abs(loss["loss"][live]).max())
    near = lambda got, want, name: np.testing.assert_array_less(np.abs(host(got) - want).max(), off * np.abs(want).max() + 1e-30, err_msg=name)
    near(learner.grad_w, grad_w, "w")
    for name, want in grads.items():
        near(learner.grad[name], want, name)
        assert (host(learner.grad[name])[host(learner.filled) == 0] == 0).all()


def test_updates_in_a_graph():
    """Forward, backward and the update of the readout, captured and replayed with eager work between: the bits of the eager steps."""
    shape = (3, 70, 2, 4, 24, 20)
    eager, graphed, other = Learner(*shape, 40, 8, 5), Learner(*shape, 40, 8, 5), Learner(*shape, 40, 8, 6)

    def step(learner):
        learner.run()
        binding.marl_muon_step(learner.w, learner.grad_w, learner.momentum, learner.w, learner.momentum, learner.ws_muon, lr=0.02)

    first = graphed.w.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(graphed)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(graphed)
    graphed.w.copy_(first)
    graphed.momentum.zero_()
    for k in range(4):
        step(eager)
        graph.replay()
        step(other)
        torch.cuda.synchronize()
        for name in eager.grad:
            assert torch.equal(eager.grad[name], graphed.grad[name]), (k, name)
        assert torch.equal(eager.loss, graphed.loss) and torch.equal(eager.w, graphed.w), k


def test_a_worker_in_a_graph():
    """The memory's step on a table, a readout, the edit of the logits and the likeliest tokens, captured once and replayed as the history grows."""
    g = gen(7)
    n, slots, H, D, V, L, K = 5, 9, 2, 24, 200, 12, 4
    q, k, v = (randn(g, 8, n, H, D).cuda() / 3 for _ in range(3))
    w = randn(g, V, H * D).cuda()
    slot = torch.randperm(slots, generator=g)[:n].to(torch.int32).cuda()
    decay, beta = torch.full((n, H), -0.1, device="cuda"), torch.full((n, H), 0.5, device="cuda")
    ones = torch.full((n,), 1.5, device="cuda")

    class Worker:
        def __init__(self):
            self.now = [torch.zeros(n, H, D, device="cuda") for _ in range(3)]
            self.table, self.o, self.logits = torch.zeros(slots, H, D, D, device="cuda"), new(n, H, D), new(n, V)
            self.history, self.length = torch.full((n, L), -1, dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")
            self.ids, self.values = new(n, K, dtype=torch.int32), new(n, K)
            self.ws = room(binding.marl_log_prob_workspace_bytes(n, V, K))

        def step(self):
            binding.marl_delta_step(*self.now, decay, beta, 1.0, slot, None, self.table, self.table, self.o)
            torch.matmul(self.o.view(n, H * D), w.t(), out=self.logits)
            binding.marl_penalize(self.logits, self.history, self.length, None, ones, ones, None, None, None, None, self.logits)
            binding.marl_log_prob(self.logits, None, None, 1.0, None, None, None, self.ids, self.values, self.ws)

        def feed(self, t):
            for to, x in zip(self.now, (q, k, v)):
                to.copy_(x[t])
            if t > 0:
                self.history[:, t - 1].copy_(self.ids[:, 0])
                self.length.fill_(t)

    eager, graphed = Worker(), Worker()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graphed.step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        graphed.step()
    graphed.table.zero_()
    for t in range(8):
        eager.feed(t)
        graphed.feed(t)
        eager.step()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(eager.ids, graphed.ids) and torch.equal(eager.logits, graphed.logits) and torch.equal(eager.table, graphed.table), t
    want = policy_oracle.log_prob(host(eager.logits), None, None, 1.0, K=K)
    assert (host(eager.ids)[:, 0] == want["top_id"][:, 0]).all()
