"""Digits that the memory and the distillation must not lose: small results of large numbers, gradients of strong decays, small remainders of a teacher, small
gradients of long rows; and calls that run at the same time."""
import numpy as np
import pytest
import torch

from oracle import memory_oracle as orc
from paper_2205_05248_amd import binding
from policy_util import DT, gen, host, near, randn

pytestmark = pytest.mark.gpu
f32 = torch.float32


def room(n):
    return torch.empty(max(n, 1), dtype=torch.uint8, device="cuda").fill_(0xff)


def new(*shape, dtype=f32):
    return torch.full(shape, float("nan"), dtype=dtype, device="cuda")


class Scan:
    """A batch on the device with all that its passes need; nothing waits before the caller does."""

    def __init__(self, q, k, v, log_decay, beta, scale, s_first=None, grad_o=None, grad_s_last=None):
        B, T, Hk, Dk = q.shape
        Hv, Dv = v.shape[2:]
        self.host = dict(q=q, k=k, v=v, log_decay=log_decay, beta=beta, s_first=s_first, grad_o=grad_o, grad_s_last=grad_s_last)
        self.scale, dt, name = scale, q.dtype, {v: k for k, v in DT.items()}[q.dtype]
        self.d = {n: None if t is None else t.cuda() for n, t in self.host.items()}
        self.o, self.s_last = new(B, T, Hv, Dv, dtype=dt), new(B, Hv, Dk, Dv)
        self.grads = [new(B, T, Hk, Dk, dtype=dt), new(B, T, Hk, Dk, dtype=dt), new(B, T, Hv, Dv, dtype=dt), new(B, T, Hv), new(B, T, Hv), new(B, Hv, Dk, Dv)]
        self.train = grad_o is not None
        self.ws = room(binding.marl_delta_scan_workspace_bytes(name, B, T, Hk, Hv, Dk, Dv, self.train))

    def forward(self):
        d = self.d
        binding.marl_delta_scan(d["q"], d["k"], d["v"], d["log_decay"], d["beta"], self.scale, None, None, d["s_first"], self.o, self.s_last, self.ws, keep=self.train)

    def backward(self):
        d = self.d
        binding.marl_delta_scan_grad(d["q"], d["k"], d["v"], d["log_decay"], d["beta"], self.scale, None, None, d["grad_o"], d["grad_s_last"], self.ws, *self.grads)

    def wanted(self):
        a = {n: None if t is None else host(t) for n, t in self.host.items()}
        memory = (a["q"], a["k"], a["v"], a["log_decay"], a["beta"], self.scale, None, None, a["s_first"])
        return orc.delta_scan(*memory)[0], orc.delta_scan_grad(*memory, a["grad_o"], a["grad_s_last"]) if self.train else None


# ------------------------------------------------------------------------------------------------ results of 16-bit types
@pytest.mark.parametrize("Dv", [16, 40])
@pytest.mark.parametrize("Dk", [16, 64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_a_small_value_in_the_place_of_a_large_one(dtype, Dk, Dv):
    """Keys are unit vectors, beta 1, no decay: an odd step puts 2^-12 of a number from 1 to 2 in the place of such a number and reads it back.  Its result is the
    sum of at most four differences that are written within a chunk: three of them rounded to 2^-24, three additions of sums below 4 to 2^-23, and as much
    again for the parts that the numbers are split into: 2^-20, which is 2^-8 of the result, on top of half a step of its type."""
    B, T, g = 64, 128, gen(Dk + Dv)
    at = (torch.arange(T // 2) % Dk).repeat_interleave(2).expand(B, T)
    k = torch.nn.functional.one_hot(at, Dk)[:, :, None].to(DT[dtype])
    v = (1 + 0.75 * torch.rand(B, T, 1, Dv, generator=g)) * torch.where(torch.rand(B, T, 1, Dv, generator=g) < 0.5, -1.0, 1.0)
    v[:, 1::2] *= 2.0 ** -12
    s = Scan(k, k, v.to(DT[dtype]), torch.zeros(B, T, 1), torch.ones(B, T, 1), 1.0)
    s.forward()
    got, want = s.o[:, 1::2], host(v.to(DT[dtype])[:, 1::2])
    near(got, want, DT[dtype], 2.0 ** -8, "o", floor=np.abs(want))


@pytest.mark.parametrize("Dv", [16, 40])
@pytest.mark.parametrize("Dk", [16, 64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_a_small_sum_over_a_state(dtype, Dk, Dv):
    """q reads two rows of the state that are each other's negative but for 2^-12 x of a number next to 1; nothing is written (beta 0) and nothing forgotten.  Rows
    of the state are fp32 numbers below 2: four roundings of their size are 2^-21, 2^-9 of the result, on top of half a step of its type."""
    B, g = 64, gen(7 * Dk + Dv)
    first = torch.zeros(B, 1, Dk, Dv)
    first[:, 0, 1] = 1 + 0.75 * torch.rand(B, Dv, generator=g)
    first[:, 0, 9] = -first[:, 0, 1] + 2.0 ** -12 * (1 + torch.rand(B, Dv, generator=g))
    q = torch.zeros(B, 3, 1, Dk)
    q[..., 1] = q[..., 9] = 1.0
    s = Scan(q.to(DT[dtype]), randn(g, B, 3, 1, Dk, dtype=DT[dtype]), randn(g, B, 3, 1, Dv, dtype=DT[dtype]), torch.zeros(B, 3, 1), torch.zeros(B, 3, 1), 1.0, first)
    s.forward()
    want = np.broadcast_to(host(first[:, :, 1]) + host(first[:, :, 9]), (B, 1, Dv))[:, None].repeat(3, 1)
    near(s.o, want, DT[dtype], 2.0 ** -9, "o", floor=np.abs(want))


# ------------------------------------------------------------------------------------------------ gradients of strong decays
# As in the tests of the delta rule: 2^-15 of the largest value for a single one, 2^-18 of the norm over all; here of the values that belong together, one
# head's or those of its steps that forget.  A decay is off by a rounding of the sum of the log decays that it stands for, 2^-24 of at most 15 to 40: less.
REL, NORM = 2.0 ** -15, 2.0 ** -18
SIZES = [(2, 64, 1, 5, 16, 16, "fp32"), (1, 150, 5, 5, 24, 40, "fp32"), (1, 100, 1, 5, 128, 72, "fp32"), (2, 130, 1, 5, 64, 33, "bf16"), (1, 140, 5, 5, 128, 128, "bf16"),
         (1, 70, 1, 5, 100, 20, "fp16")]


def random_scan(B, T, Hk, Hv, Dk, Dv, dtype, seed, log_decay=None):
    g = gen(seed)
    unit = lambda t: (t / t.norm(dim=-1, keepdim=True)).to(DT[dtype])
    values = lambda: randn(g, B, T, Hv, Dv, dtype=DT[dtype])
    log_decay = -0.1 * torch.rand(B, T, Hv, generator=g) if log_decay is None else log_decay(torch.rand(B, T, Hv, generator=g))
    return Scan(unit(randn(g, B, T, Hk, Dk)), unit(randn(g, B, T, Hk, Dk)), values(), log_decay, torch.rand(B, T, Hv, generator=g), Dk ** -0.5,
                randn(g, B, Hv, Dk, Dv) * 0.5, values(), randn(g, B, Hv, Dk, Dv) * 0.5)


def same_digits(got, want, name):
    assert np.abs(got - want).max() <= REL * np.abs(want).max(), (name, np.abs(got - want).max() / np.abs(want).max())
    assert np.linalg.norm(got - want) <= NORM * np.linalg.norm(want), (name, np.linalg.norm(got - want) / np.linalg.norm(want))


@pytest.mark.parametrize("size", SIZES)
def test_the_gradient_of_a_head_that_forgets_at_once(size):
    """Every head has a decay of its own strength, and with it a gradient of its own size: down to e^-40 of the others'."""
    strength = torch.tensor([0.5, 8.0, 12.0, 15.0, 40.0])
    s = random_scan(*size, sum(size[:6]), lambda r: -strength * (0.9 + 0.1 * r))
    s.forward()
    s.backward()
    got, want = host(s.grads[3]), s.wanted()[1][3]
    for h in range(5):
        same_digits(got[:, :, h], want[:, :, h], f"head {h}")


@pytest.mark.parametrize("size", SIZES)
def test_the_gradient_of_a_step_that_forgets(size):
    """Strong decays between weak ones: their gradients are as small as what they leave of the state."""
    hard = torch.arange(size[1]) % 5 == 3
    s = random_scan(*size, 1 + sum(size[:6]), lambda r: torch.where(hard[None, :, None], -12.0 - r, -0.1 * r))
    s.forward()
    s.backward()
    got, want = host(s.grads[3]), s.wanted()[1][3]
    for name, steps in (("hard", hard.numpy()), ("soft", ~hard.numpy())):
        same_digits(got[:, steps], want[:, steps], name)


# ------------------------------------------------------------------------------------------------ distillation
# Gradients are compared with the sizes of their own terms, W q and p, or W q and p_r q / q_r.  An exponent is made of z (|z| <= 32, rounded: 2^-19), log_sum (1.25 x
# 2^-18, as in the tests of the distillation), their difference (2^-20) and its product with log2 e (36 x 2^-24 at |z - log_sum| <= 25): 2.6 x 2^-18 of q.  q / q_r has
# log_rest's 2.5 x 2^-18 on top, and q_r itself |log_rest| <= 25 times 2^-24: 5.7 x 2^-18 in all, where the remainder p_r is as exact as the alternatives are.
TERMS = 5.7 * 2.0 ** -18


def distill(s, scale, K):
    R, V = s["logits"].shape
    logits, ids, values = s["logits"].cuda(), s["top_id"].cuda(), s["top_value"].cuda()
    avail = None if s.get("avail") is None else s["avail"].cuda()
    loss, log_sum, rest, grad = new(R), new(R), new(R), new(R, V, dtype=logits.dtype)
    tail = s["tail"]
    binding.marl_distill(logits, ids, values, avail, scale, tail, loss, log_sum, rest if tail else None, room(binding.marl_distill_workspace_bytes(R, V, K)))
    binding.marl_distill_grad(logits, ids, values, avail, scale, tail, log_sum, rest if tail else None, s["grad_loss"].cuda(), grad)
    with np.errstate(invalid="ignore"):
        want = orc.distill(host(s["logits"]), host(s["top_id"]), host(s["top_value"]), None if s.get("avail") is None else host(s["avail"]), scale, tail, host(s["grad_loss"]))
    return loss, grad, want


# What a teacher is sure of: log probabilities of its alternatives.
SURE = {"1e-4": [-1e-4], "1e-6": [-1e-6], "1e-7": [-1e-7], "three": [float(np.log(0.97)), float(np.log(0.02)), float(np.log(0.009995))],
        "two_halves": [float(np.log(0.5)) - 1e-6, float(np.log(0.5)) - 2e-6], "sure": [0.0]}


@pytest.mark.parametrize("V", [40, 200, 600, 3000, 40000])
@pytest.mark.parametrize("values", SURE)
def test_the_small_remainder_of_a_sure_teacher(values, V):
    """A student that is sure too (its other places hold e^-10 to e^-20) feels the remainder alone at all other places."""
    values, R, g = SURE[values], 9, gen(V)
    K = len(values)
    s = dict(logits=randn(g, R, V), tail=True, grad_loss=randn(g, R), top_value=torch.tensor(values).expand(R, K).contiguous())
    s["top_id"] = torch.stack([torch.randperm(V, generator=g)[:K] for _ in range(R)]).to(torch.int32)
    s["logits"].scatter_(1, s["top_id"].long(), 20.0)
    loss, grad, want = distill(s, 1.0, K)
    near(grad, want["grad"], f32, TERMS, "grad", floor=want["grad_size"])
    near(loss, want["loss"], f32, 4 * 1.25 * 2.0 ** -18, "loss", floor=np.maximum(1.0, np.abs(want["loss"])))


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("R,V,K", [(9, 40, 5), (7, 257, 20), (6, 2048, 64), (5, 2049, 20), (4, 8192, 50), (3, 8193, 1), (2, 50021, 20), (1, 140001, 64)])
def test_every_gradient_of_a_row(R, V, K, dtype, tail):
    """Against the size of its own terms, so that none of the many small ones of a long row could be left out."""
    g = gen(R + V + K)
    s = dict(logits=randn(g, R, V, dtype=DT[dtype]), tail=tail, avail=None, grad_loss=(0.5 + torch.rand(R, generator=g)) * (4096.0 if dtype == "fp16" else 1.0))
    s["top_id"] = torch.stack([torch.randperm(V, generator=g)[:K] for _ in range(R)]).to(torch.int32)
    s["top_value"] = torch.log(0.8 * torch.softmax(randn(g, R, K), 1))
    if V % 2:
        s["avail"] = (torch.rand(R, V, generator=g) < 0.7).to(torch.uint8)
    _, grad, want = distill(s, 0.8, K)
    near(grad, want["grad"], DT[dtype], TERMS, "grad", floor=want["grad_size"])
    there = want["grad_size"] > 0
    step = torch.finfo(DT[dtype]).smallest_normal * torch.finfo(DT[dtype]).eps
    assert (np.abs(want["grad"])[there] > 2 * (TERMS * want["grad_size"][there] + step)).mean() > 0.999


# ------------------------------------------------------------------------------------------------ at the same time
def side_by_side(calls):
    """Every call alone, then all of them on streams of their own, over and over without a wait: the outputs of both."""
    alone = []
    for call, outs in calls:
        call()
        torch.cuda.synchronize()
        alone.append([t.clone() for t in outs])
        for t in outs:
            t.fill_(7)
    streams = [torch.cuda.Stream() for _ in calls]
    torch.cuda.synchronize()
    for _ in range(6):
        for stream, (call, _) in zip(streams, calls):
            with torch.cuda.stream(stream):
                call()
    torch.cuda.synchronize()
    for (_, outs), want in zip(calls, alone):
        for got, w in zip(outs, want):
            assert torch.equal(got, w)


@pytest.mark.parametrize("size", [(4, 300, 1, 2, 64, 64, "bf16"), (8, 200, 2, 2, 16, 16, "fp32"), (2, 300, 1, 4, 128, 128, "bf16")])
def test_scans_at_the_same_time(size):
    sets = [random_scan(*size, 50 + i) for i in range(2)]

    def call(s):
        s.forward()
        s.backward()

    side_by_side([(lambda s=s: call(s), [s.o, s.s_last, *s.grads]) for s in sets])


@pytest.mark.parametrize("R,V", [(300, 40), (40, 30001)])
def test_distillations_at_the_same_time(R, V):
    calls, K = [], 9
    for i in range(2):
        g = gen(60 + i)
        logits = randn(g, R, V).cuda()
        ids = torch.stack([torch.randperm(V, generator=g)[:K] for _ in range(R)]).to(torch.int32).cuda()
        values, upstream = torch.log(0.9 * torch.softmax(randn(g, R, K), 1)).cuda(), randn(g, R).cuda()
        loss, log_sum, rest, grad = new(R), new(R), new(R), new(R, V)
        bytes_ = binding.marl_distill_workspace_bytes(R, V, K)
        assert (bytes_ > 0) == (V > 2048)
        ws = room(bytes_)

        def call(logits=logits, ids=ids, values=values, upstream=upstream, loss=loss, log_sum=log_sum, rest=rest, grad=grad, ws=ws):
            binding.marl_distill(logits, ids, values, None, 1.0, True, loss, log_sum, rest, ws)
            binding.marl_distill_grad(logits, ids, values, None, 1.0, True, log_sum, rest, upstream, grad)

        calls.append((call, [loss, log_sum, rest, grad]))
    side_by_side(calls)
