"""Distillation from kept alternatives on the GPU against the 64-bit oracle.

Tolerance.  With |z| <= Z = 32 an exponent is off by at most Z 2^-23 (z rounded, its distance to the maximum rounded), and so is every
probability, every sum of them, log_sum and log_rest by that part of itself; hardware exponentials and the order of sums add a few
2^-23: 2^-18 and a quarter of it, as for the log probabilities.  The loss is a sum of p (log p - log q) with sum p <= 1: the same amount
absolutely, twice with the other places' part, plus the rounding of p and log p themselves (|log p| < 16): 4 x that in all.  p_r = 1 - sum p
is off by K 2^-24 at most, and multiplies a logarithm of at most 16: below that too.  A gradient is the difference of two probabilities: each off by
1.25 x 2^-18 of itself, and W q_r - p_r by the same of its terms.
"""
import numpy as np
import pytest
import torch

from oracle import memory_oracle as orc
from paper_2205_05248_amd import binding
from policy_util import DT, gen, host, near, randn

pytestmark = pytest.mark.gpu
REL = 1.25 * 2.0 ** -18
f32 = torch.float32


def make(R, V, K, dtype, seed, avail="none", ld=None, far=0.0):
    g = gen(seed)
    s = dict(V=V, logits=(randn(g, R, ld or V) * 3).to(DT[dtype]), avail=None)
    if avail == "rows":
        s["avail"] = (torch.rand(R, ld or V, generator=g) < 0.6).to(torch.uint8)
        s["avail"][R // 2] = 0
        s["logits"][:, :V][s["avail"][:, :V] == 0] = float("nan")
    elif avail == "shared":
        s["avail"] = (torch.rand(V, generator=g) < 0.6).to(torch.uint8)
        s["avail"][V - 1] = 1
        s["logits"][:, :V][:, s["avail"] == 0] = float("inf")
    s["top_id"] = torch.stack([torch.randperm(V, generator=g)[:K] if V >= K else torch.randint(0, V, (K,), generator=g) for _ in range(R)]).to(torch.int32)
    s["top_id"][torch.rand(R, K, generator=g) < 0.1] = -1
    s["top_id"][R // 3] = -1                                       # a row without an alternative
    p = torch.softmax(randn(g, R, K) * 1.5, 1) * 0.9
    s["top_value"] = torch.log(p)
    if far:
        s["logits"][:, :V].scatter_(1, s["top_id"].long().clamp(min=0), far)
    s["grad_loss"] = randn(g, R)
    return s


def run(s, scale, tail, in_place=False):
    V, R = s["V"], s["logits"].shape[0]
    K = s["top_id"].shape[1]
    wide = s["logits"].cuda()
    logits = wide[:, :V]
    avail = None if s["avail"] is None else s["avail"].cuda()[..., :V]
    nan = float("nan")
    o = {k: torch.full((R,), nan, device="cuda") for k in ("loss", "log_sum", "log_rest")}
    ids, values = s["top_id"].cuda(), s["top_value"].cuda()
    ws = torch.empty(binding.marl_distill_workspace_bytes(R, V, K), dtype=torch.uint8, device="cuda").fill_(0xff)
    binding.marl_distill(logits, ids, values, avail, scale, tail, o["loss"], o["log_sum"], o["log_rest"] if tail else None, ws)
    out = logits if in_place else torch.full((R, V), nan, dtype=logits.dtype, device="cuda")
    binding.marl_distill_grad(logits, ids, values, avail, scale, tail, o["log_sum"], o["log_rest"] if tail else None, s["grad_loss"].cuda(), out)
    torch.cuda.synchronize()
    if in_place and wide.shape[1] > V:
        assert torch.equal(wide[:, V:].cpu(), s["logits"][:, V:])
    o["grad"] = out
    return o


def check(s, o, scale, tail):
    V = s["V"]
    logits = host(s["logits"][:, :V])
    with np.errstate(invalid="ignore"):
        want = orc.distill(logits, host(s["top_id"]), host(s["top_value"]), None if s["avail"] is None else host(s["avail"][..., :V]), scale, tail,
                           host(s["grad_loss"]))
    finite = logits[np.isfinite(logits)]
    rel = REL * max(1.0, scale * np.abs(finite).max(initial=0.0) / 32)
    near(o["loss"], want["loss"], f32, 4 * rel, "loss", floor=np.maximum(1.0, np.abs(want["loss"])))
    near(o["log_sum"], want["log_sum"], f32, rel, "log_sum", floor=1.0)
    if tail:
        near(o["log_rest"], want["log_rest"], f32, 2 * rel, "log_rest", floor=1.0)
    floor = scale * np.abs(host(s["grad_loss"]))[:, None]
    near(o["grad"], want["grad"], o["grad"].dtype, 4 * rel, "grad", floor=np.broadcast_to(floor, want["grad"].shape))


SIZES = [(1, 1, 1), (3, 2, 2), (9, 16, 3), (65, 40, 5), (33, 60, 50), (20, 200, 20), (7, 257, 64), (10, 500, 5), (6, 2048, 64), (5, 2049, 20),
         (4, 8192, 50), (3, 8193, 1), (2, 50021, 20), (1, 140001, 64)]


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("dtype,avail", [("fp32", "none"), ("bf16", "rows"), ("fp16", "shared")])
@pytest.mark.parametrize("size", SIZES)
def test_distill(size, dtype, avail, tail):
    R, V, K = size
    s = make(R, V, K, dtype, sum(size), avail)
    check(s, run(s, 0.8, tail), 0.8, tail)


@pytest.mark.parametrize("V,K", [(40, 5), (300, 10), (5001, 7)])
@pytest.mark.parametrize("in_place", [False, True])
def test_wider_rows_and_in_place(V, K, in_place):
    for dtype, avail in (("fp32", "rows"), ("bf16", "none")):
        s = make(21, V, K, dtype, V, avail, ld=V + 13)
        check(s, run(s, 1.0, True, in_place), 1.0, True)


@pytest.mark.parametrize("V", [40, 5000])
def test_rows_behind_32_bits(V):
    R, K, ld = 3, 6, (1 << 31) + 24
    s = make(R, V, K, "fp16", V + 1)
    far = torch.empty(2 * ld + V, dtype=torch.float16, device="cuda").as_strided((R, V), (ld, 1))
    far.copy_(s["logits"])
    ids, values, o = s["top_id"].cuda(), s["top_value"].cuda(), {k: torch.empty(R, device="cuda") for k in ("loss", "log_sum", "log_rest")}
    ws = torch.empty(binding.marl_distill_workspace_bytes(R, V, K), dtype=torch.uint8, device="cuda")
    binding.marl_distill(far, ids, values, None, 0.8, True, o["loss"], o["log_sum"], o["log_rest"], ws)
    binding.marl_distill_grad(far, ids, values, None, 0.8, True, o["log_sum"], o["log_rest"], s["grad_loss"].cuda(), far)
    check(s, {**o, "grad": far}, 0.8, True)


@pytest.mark.parametrize("V", [40, 5000])
def test_an_index_listed_twice_counts_twice(V):
    s = make(12, V, 6, "fp32", 5)
    s["top_id"][:, 3] = s["top_id"][:, 0]
    s["top_id"][:, 5] = s["top_id"][:, 0]
    for tail in (False, True):
        check(s, run(s, 1.0, tail), 1.0, tail)


@pytest.mark.parametrize("V,K", [(5, 5), (64, 64)])
def test_every_place_kept(V, K):
    """No place is left for the teacher's remainder, which then counts for nothing."""
    s = make(30, V, K, "fp32", 6)
    s["top_id"] = torch.stack([torch.randperm(V, generator=gen(i))[:K] for i in range(30)]).to(torch.int32)
    check(s, run(s, 1.0, True), 1.0, True)


@pytest.mark.parametrize("far", [60.0, -60.0])
@pytest.mark.parametrize("V", [40, 3000])
def test_all_or_nothing_at_the_kept_places(V, far):
    """The student has all of its probability at the kept places, or all but e^-60 of it at the others: log_rest and the loss stay exact."""
    s = make(16, V, 4, "fp32", 7, far=far)
    s["top_id"][s["top_id"] < 0] = 0
    for tail in (False, True):
        check(s, run(s, 2.0, tail), 2.0, tail)


def test_teacher_certain_or_without_probability():
    s = make(8, 50, 4, "fp32", 8)
    s["top_value"][:4] = torch.tensor([0.0, -float("inf"), -float("inf"), -float("inf")])
    s["top_value"][4] = -float("inf")
    s["top_value"][5] = torch.log(torch.tensor([0.5, 0.3, 0.2, 0.1]))          # more than 1 in all
    for tail in (False, True):
        check(s, run(s, 1.0, tail), 1.0, tail)


@pytest.mark.parametrize("V", [40, 600, 4000])
def test_what_is_not_finite_stays_in_its_row(V):
    s = make(8, V, 4, "fp32", 9)
    s["top_id"][:] = torch.tensor([1, 3, 5, 7], dtype=torch.int32)
    s["logits"][1, 2] = float("nan")
    s["logits"][2, 3] = float("inf")
    s["logits"][3, 5] = -float("inf")                              # a kept place without probability is left out
    s["top_value"][4, 1] = float("nan")
    s["top_value"][5, 1] = float("inf")
    s["grad_loss"][1] = 0.0                                        # its gradient is 0 although its loss is NaN
    for tail in (False, True):
        o = run(s, 1.0, tail)
        loss, grad = host(o["loss"]), host(o["grad"])
        bad = np.isin(np.arange(8), [1, 2, 4, 5])
        assert np.isnan(loss[bad]).all() and np.isfinite(loss[~bad]).all()
        assert (grad[1] == 0).all() and np.isnan(grad[4]).all() and np.isnan(grad[5]).all()
        assert np.isnan(grad[2]).all()
        assert np.isfinite(grad[~bad]).all()
        keep = torch.tensor([0, 3, 6, 7])
        part = {k: (v[keep] if torch.is_tensor(v) else v) for k, v in s.items()}
        check(part, {k: v[keep.cuda()] for k, v in o.items()}, 1.0, tail)


def test_a_scale_that_takes_a_logit_to_nothing():
    s = make(4, 40, 3, "fp32", 10)
    s["logits"][:, 5] = -3e38
    s["top_id"][:] = torch.tensor([5, 1, 2], dtype=torch.int32)
    o = run(s, 2.0, True)
    s["logits"][:, 5] = -float("inf")
    check(s, o, 2.0, True)


def test_of_the_teachers_own_alternatives():
    """What marl_log_prob writes is what this reads: a student that is its teacher has no loss and no gradient."""
    g = gen(11)
    logits = (randn(g, 30, 5000) * 3).cuda()
    K = 20
    logp = [torch.empty(30, device="cuda") for _ in range(2)]
    ids, values = torch.empty(30, K, dtype=torch.int32, device="cuda"), torch.empty(30, K, device="cuda")
    ws = torch.empty(binding.marl_log_prob_workspace_bytes(30, 5000, K), dtype=torch.uint8, device="cuda")
    binding.marl_log_prob(logits, None, None, 0.7, None, None, logp[0], ids, values, ws)
    ws = torch.empty(binding.marl_distill_workspace_bytes(30, 5000, K), dtype=torch.uint8, device="cuda")
    loss, log_sum, rest = (torch.empty(30, device="cuda") for _ in range(3))
    binding.marl_distill(logits, ids, values, None, 0.7, True, loss, log_sum, rest, ws)
    assert float((log_sum - logp[0]).abs().max()) <= 2 * REL
    assert float(loss.abs().max()) <= 4 * REL
    grad = torch.empty_like(logits)
    binding.marl_distill_grad(logits, ids, values, None, 0.7, True, log_sum, rest, torch.ones(30, device="cuda"), grad)
    assert float(grad.abs().max()) <= 4 * REL


@pytest.mark.parametrize("V", [40, 9000])
def test_graph(V):
    sets = [make(20, V, 5, "fp32", 20 + i) for i in range(3)]
    eager = [run(s, 1.0, True) for s in sets]
    names = ("logits", "top_id", "top_value", "grad_loss")
    d = {n: sets[0][n].cuda().clone() for n in names}
    out = {n: torch.zeros_like(t) for n, t in eager[0].items()}
    ws = torch.empty(binding.marl_distill_workspace_bytes(20, V, 5), dtype=torch.uint8, device="cuda")

    def once():
        binding.marl_distill(d["logits"], d["top_id"], d["top_value"], None, 1.0, True, out["loss"], out["log_sum"], out["log_rest"], ws)
        binding.marl_distill_grad(d["logits"], d["top_id"], d["top_value"], None, 1.0, True, out["log_sum"], out["log_rest"], d["grad_loss"], out["grad"])

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        once()
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        once()
    for i in (1, 2, 0):
        for n in names:
            d[n].copy_(sets[i][n])
        graph.replay()
        torch.cuda.synchronize()
        for n, t in eager[i].items():
            assert torch.equal(out[n], t), (i, n)
        run(sets[i], 1.0, True)
