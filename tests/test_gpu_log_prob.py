"""Log probabilities, entropy, alternatives and the logits' gradient on the GPU against the 64-bit oracle.

Tolerance.  z = scale * logit is rounded once and its distance to the maximum once more: at |z| <= Z an exponent is off by
at most Z * 2^-23, and so is every p by that part of itself, the sum by that part and log_sum by that much (plus its own
rounding, Z 2^-24); the hardware exponential and the order of the sum add a few 2^-23.  With Z <= 32: 2^-18 plus a
quarter of it.  The entropy adds p |z - m| of the same parts, |z - m| <= 2 Z: 64 times 2^-18 would be the bound
for all of the mass at the far end; where the mass is, |log p| <= log V < 12, which gives 12 * 2^-18.  A gradient is a sum of terms with such parts: it is
held to four times 2^-18 of its terms' sizes (p, the entropy, the difference and the products).
"""
import numpy as np
import pytest
import torch

from oracle import policy_oracle as orc
from policy_util import DT, gen, host, near, randn
from paper_2205_05248_amd import binding

pytestmark = pytest.mark.gpu
REL = 1.25 * 2.0 ** -18
f32 = torch.float32


def make(R, V, dtype, seed, avail="none", ld=None, ld_avail=None):
    g = gen(seed)
    wide = randn(g, R, ld or V) * 3
    s = dict(logits=wide.to(DT[dtype]), V=V, token=torch.randint(0, V, (R,), generator=g).to(torch.int32), avail=None)
    if avail == "rows":
        a = (torch.rand(R, ld_avail or V, generator=g) < 0.6).to(torch.uint8)
        a[R // 2] = 0                                              # a row with nothing
        s["avail"] = a
        s["logits"][:, :V][a[:, :V] == 0] = float("nan")
    elif avail == "shared":
        a = (torch.rand(V, generator=g) < 0.6).to(torch.uint8)
        a[V - 1] = 1
        s["avail"] = a
        s["logits"][:, :V][:, a == 0] = float("inf")
    s["grad_logp"], s["grad_entropy"] = randn(g, R), randn(g, R)
    return s


def run(s, scale, K, grad=True, in_place=False, parts=("logp", "entropy")):
    V, R = s["V"], s["logits"].shape[0]
    wide = s["logits"].cuda()
    logits = wide[:, :V]
    token = s["token"].cuda()
    avail = None if s["avail"] is None else s["avail"].cuda()
    if avail is not None and avail.dim() == 2:
        avail = avail[:, :V]
    nan = float("nan")
    o = {k: torch.full((R,), nan, device="cuda") for k in ("logp", "entropy", "log_sum")}
    if K:
        o.update(top_id=torch.full((R, K), -7, dtype=torch.int32, device="cuda"), top_logp=torch.full((R, K), nan, device="cuda"))
    ws = torch.empty(binding.marl_log_prob_workspace_bytes(R, V, K), dtype=torch.uint8, device="cuda").fill_(0xff)
    binding.marl_log_prob(logits, token, avail, scale, o["logp"], o["entropy"], o["log_sum"], o.get("top_id"), o.get("top_logp"), ws)
    if grad:
        out = logits if in_place else torch.full((R, V), nan, dtype=logits.dtype, device="cuda")
        binding.marl_log_prob_grad(logits, token, avail, scale, o["log_sum"], o["entropy"], s["grad_logp"].cuda() if "logp" in parts else None,
                                   s["grad_entropy"].cuda() if "entropy" in parts else None, out)
        o["grad"] = out
        if in_place and wide.shape[1] > V:
            assert torch.equal(wide[:, V:].cpu(), s["logits"][:, V:])
    torch.cuda.synchronize()
    return o


def check(s, o, scale, K, parts=("logp", "entropy")):
    V = s["V"]
    logits, token = host(s["logits"][:, :V]), host(s["token"])
    avail = None if s["avail"] is None else host(s["avail"][..., :V])
    want = orc.log_prob(logits, token, avail, scale, K)
    finite = logits[np.isfinite(logits) & (np.abs(logits) < 1e30)]
    rel = REL * max(1.0, scale * np.abs(finite).max(initial=0.0) / 32)     # the derivation's Z
    near(o["logp"], want["logp"], f32, 0, "logp", floor=0) if V == 1 else near(o["logp"], want["logp"], f32, rel, "logp", floor=1.0)
    near(o["log_sum"], want["log_sum"], f32, rel, "log_sum", floor=1.0)
    near(o["entropy"], want["entropy"], f32, 12 * rel, "entropy", floor=1.0)
    if K:
        assert np.array_equal(host(o["top_id"]), want["top_id"])
        near(o["top_logp"], want["top_logp"], f32, rel, "top_logp", floor=1.0)
    if "grad" in o:
        grad = orc.log_prob_grad(logits, token, avail, scale, host(s["grad_logp"]) if "logp" in parts else None,
                                 host(s["grad_entropy"]) if "entropy" in parts else None)
        near(o["grad"], grad, s["logits"].dtype, 4 * rel, "grad", floor=terms(s, logits, avail, scale, want, parts))


def terms(s, logits, avail, scale, want, parts):
    """Sizes of the terms that a gradient is the sum of: 1 - p and log p + entropy cancel, what they are made of does not."""
    with np.errstate(invalid="ignore", over="ignore", under="ignore"):
        lp = scale * logits - want["log_sum"][:, None]
        ok = np.isfinite(lp) if avail is None else np.isfinite(lp) & (avail != 0)
        lp = np.where(ok, lp, 0.0)
        p = np.where(ok, np.exp(lp), 0.0)
    size = np.zeros(p.shape)
    if "logp" in parts:
        taken = np.arange(s["V"])[None] == host(s["token"])[:, None]
        size += np.abs(host(s["grad_logp"]))[:, None] * (taken + p)
    if "entropy" in parts:
        size += np.abs(host(s["grad_entropy"]))[:, None] * p * (np.abs(lp) + want["entropy"][:, None])
    return scale * size


SIZES = [(1, 1), (5, 2), (24, 9), (33, 40), (7, 64), (6, 65), (9, 130), (5, 257), (3, 1000), (4, 4096), (2, 5001), (3, 20003), (2, 70000)]


@pytest.mark.parametrize("R,V", SIZES)
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("avail", ["none", "rows", "shared"])
def test_forward_and_backward(R, V, dtype, avail):
    k = SIZES.index((R, V))
    K = (0, 1, 5, 20, 64)[k % 5]
    odd = {"rows": V + 3, "none": None, "shared": V + 1}[avail]
    s = make(R, V, dtype, 100 + k, avail, odd, odd)
    scale = (1.0, 0.7, 1.3)[k % 3]
    check(s, run(s, scale, K), scale, K)


@pytest.mark.parametrize("parts", [("logp",), ("entropy",), ()])
def test_gradients_of_one_part(parts):
    s = make(6, 300, "fp32", 3, "rows")
    check(s, run(s, 1.0, 0, parts=parts), 1.0, 0, parts)


@pytest.mark.parametrize("V,dtype,ld", [(40, "fp32", 40), (333, "bf16", 340), (9001, "fp16", 9001)])
def test_gradient_in_place(V, dtype, ld):
    s = make(20, V, dtype, 4, "none", ld)
    check(s, run(s, 1.0, 0, in_place=True), 1.0, 0)


def test_tokens_out_of_range_and_masked():
    s = make(5, 12, "fp32", 5, "rows")
    s["avail"][0], s["avail"][1], s["avail"][3] = 1, 1, 1
    s["logits"] = torch.nan_to_num(s["logits"])
    s["token"][0], s["token"][1] = -1, 12
    s["token"][3] = 4
    s["avail"][3, 4] = 0
    o = run(s, 1.0, 3)
    check(s, o, 1.0, 3)
    assert o["logp"][0] == 0 and o["logp"][1] == 0 and o["logp"][3] == -float("inf")


@pytest.mark.parametrize("V", [7, 900, 30000])
def test_infinities(V):
    s = make(4, V, "fp32", 6)
    s["logits"][0] = -float("inf")                                 # nothing available
    s["logits"][1, ::2] = -float("inf")
    s["token"][1], s["token"][0] = 0, 1                            # a token without probability
    low = torch.finfo(f32).min
    s["logits"][2] = low
    s["logits"][2, V // 2] = 0.0                                   # the type's lowest value everywhere else
    s["token"][2] = V // 2
    o = run(s, 1.0, 4)
    check(s, o, 1.0, 4)
    assert o["logp"][0] == 0 and o["logp"][2] == 0 and not o["grad"][0].any()


@pytest.mark.parametrize("V", [7, 900, 30000])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_an_available_nan_or_infinity_stays_in_its_row(V, value):
    s = make(3, V, "fp32", 7)
    clean = run(s, 1.0, 3)
    s["logits"][1, V - 2] = value
    o = run(s, 1.0, 3)
    for k in ("logp", "entropy", "log_sum"):
        assert torch.isnan(o[k][1]) and torch.equal(o[k][::2], clean[k][::2]), k
    assert torch.equal(o["top_id"][::2], clean["top_id"][::2]) and torch.equal(o["grad"][::2], clean["grad"][::2])
    assert (o["top_id"][1] >= -1).all() and (o["top_id"][1] < V).all()


@pytest.mark.parametrize("V,K", [(50, 50), (50, 64), (3000, 64), (40000, 64)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_ties_go_to_the_lowest_index(V, K, dtype):
    g = gen(V)
    s = make(4, V, dtype, 8)
    s["logits"] = torch.randint(-3, 3, (4, V), generator=g).to(DT[dtype])
    s["logits"][1] = 0.0
    s["logits"][2] = torch.arange(V).to(DT[dtype]) / 4             # ascending: every entry is a new best
    s["logits"][3, ::2] *= -1                                      # -0 and +0 are equal
    check(s, run(s, 1.0, K), 1.0, K)


def test_outputs_may_be_left_out():
    s = make(3, 100, "bf16", 9)
    logits = s["logits"].cuda()
    lone = torch.empty(3, device="cuda")
    ws = torch.empty(max(1, binding.marl_log_prob_workspace_bytes(3, 100, 0)), dtype=torch.uint8, device="cuda")
    binding.marl_log_prob(logits, None, None, 1.0, None, None, lone, workspace=ws)
    torch.cuda.synchronize()
    near(lone, orc.log_prob(host(s["logits"]), None, None, 1.0)["log_sum"], f32, REL, "log_sum", floor=1.0)


def test_rows_beyond_thirty_two_bits():
    """Two rows whose distance does not fit 32 bits."""
    ld = (1 << 31) + 128
    wide = torch.empty(ld + 1000, dtype=torch.bfloat16, device="cuda")
    rows = torch.as_strided(wide, (2, 1000), (ld, 1))
    rows.copy_(randn(gen(10), 2, 1000, dtype=torch.bfloat16))
    s = dict(logits=rows.cpu(), V=1000, token=torch.tensor([3, 999], dtype=torch.int32), avail=None, grad_logp=torch.ones(2), grad_entropy=torch.ones(2))
    o = {k: torch.empty(2, device="cuda") for k in ("logp", "entropy", "log_sum")}
    ws = torch.empty(max(1, binding.marl_log_prob_workspace_bytes(2, 1000, 0)), dtype=torch.uint8, device="cuda")
    token, one = s["token"].cuda(), torch.ones(2, device="cuda")
    binding.marl_log_prob(rows, token, None, 1.0, o["logp"], o["entropy"], o["log_sum"], workspace=ws)
    binding.marl_log_prob_grad(rows, token, None, 1.0, o["log_sum"], o["entropy"], one, one, rows)
    torch.cuda.synchronize()
    o["grad"] = rows.contiguous()
    check(s, o, 1.0, 0)


@pytest.mark.parametrize("R,V,K", [(300, 40, 5), (2, 60000, 20)])
def test_replayed_from_a_graph_and_on_another_stream(R, V, K):
    s = make(R, V, "fp32", 11)
    logits, token = s["logits"].cuda(), s["token"].cuda()
    gl, ge = s["grad_logp"].cuda(), s["grad_entropy"].cuda()

    def fresh():
        o = [torch.zeros(R, device="cuda") for _ in range(3)]
        return o + [torch.zeros(R, K, dtype=torch.int32, device="cuda"), torch.zeros(R, K, device="cuda"), torch.zeros(R, V, device="cuda"),
                    torch.empty(binding.marl_log_prob_workspace_bytes(R, V, K), dtype=torch.uint8, device="cuda")]

    def go(o):
        binding.marl_log_prob(logits, token, None, 1.0, o[0], o[1], o[2], o[3], o[4], o[6])
        binding.marl_log_prob_grad(logits, token, None, 1.0, o[2], o[1], gl, ge, o[5])

    got = fresh()
    go(got)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go(got)
    side = torch.cuda.Stream()
    for k in range(3):
        logits.mul_(0.9)
        want = fresh()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            go(want)
        side.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got[:6], want[:6]):
            assert torch.equal(a, b), k


@pytest.mark.parametrize("V", [8187, 8192, 8193, 16384, 18437])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("shift", [0, 1, 3])
@pytest.mark.parametrize("avail", ["none", "rows"])
def test_long_rows_that_begin_anywhere(V, dtype, shift, avail):
    """Ends of a row on either side of a workgroup's pieces, rows and outputs at differing alignments; nothing beside the row is
    read into it or written."""
    s = make(5, V, dtype, 12 + shift, avail)
    R, ld = 5, V + 5
    wide = torch.full((R, ld), 1e4, dtype=DT[dtype], device="cuda")    # what a read beside the row would find
    logits = wide[:, shift:shift + V]
    logits.copy_(s["logits"])
    avail_t = None if s["avail"] is None else s["avail"].cuda()
    token = s["token"].cuda()
    o = {k: torch.empty(R, device="cuda") for k in ("logp", "entropy", "log_sum")}
    ws = torch.empty(max(1, binding.marl_log_prob_workspace_bytes(R, V, 0)), dtype=torch.uint8, device="cuda")
    out = torch.full((R, V + 2), 7.0, dtype=DT[dtype], device="cuda")
    binding.marl_log_prob(logits, token, avail_t, 1.1, o["logp"], o["entropy"], o["log_sum"], workspace=ws)
    binding.marl_log_prob_grad(logits, token, avail_t, 1.1, o["log_sum"], o["entropy"], s["grad_logp"].cuda(), s["grad_entropy"].cuda(), out[:, 1:V + 1])
    torch.cuda.synchronize()
    assert (out[:, 0] == 7).all() and (out[:, V + 1] == 7).all()
    o["grad"] = out[:, 1:V + 1].contiguous()
    check(s, o, 1.1, 0)


@pytest.mark.parametrize("V", [1, 3, 16, 17, 40, 63, 64, 65, 200, 255, 256])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("avail", ["none", "rows", "shared"])
@pytest.mark.parametrize("in_place", [False, True])
def test_short_rows_without_gaps(V, dtype, avail, in_place):
    """Full and partial waves, tensors that begin anywhere; nothing beside them is read into a row or written."""
    for R, shift in ((1, 0), (67, 1), (129, 3)):
        s = make(R, V, dtype, 13, avail)
        whole = torch.full((R * V + 32,), 1e4, dtype=DT[dtype], device="cuda")
        logits = whole[16 + shift:16 + shift + R * V].view(R, V)
        logits.copy_(s["logits"])
        avail_t = None
        if s["avail"] is not None:
            bytes_ = torch.zeros(s["avail"].numel() + 32, dtype=torch.uint8, device="cuda")
            avail_t = bytes_[5 + shift:5 + shift + s["avail"].numel()].view(s["avail"].shape)
            avail_t.copy_(s["avail"])
        token = s["token"].cuda()
        o = {k: torch.empty(R, device="cuda") for k in ("logp", "entropy", "log_sum")}
        binding.marl_log_prob(logits, token, avail_t, 0.9, o["logp"], o["entropy"], o["log_sum"])
        room = whole if in_place else torch.full((R * V + 32,), 1e4, dtype=DT[dtype], device="cuda")
        lead = 16 + shift if in_place else 16
        grad = room[lead:lead + R * V].view(R, V)
        binding.marl_log_prob_grad(logits, token, avail_t, 0.9, o["log_sum"], o["entropy"], s["grad_logp"].cuda(), s["grad_entropy"].cuda(), grad)
        torch.cuda.synchronize()
        beside = torch.full((), 1e4, dtype=DT[dtype], device="cuda")
        assert (room[:lead] == beside).all() and (room[lead + R * V:] == beside).all()
        o["grad"] = grad.clone()
        check(s, o, 0.9, 0)



@pytest.mark.parametrize("V", [513, 1000, 2048])
@pytest.mark.parametrize("K", [62, 63, 64])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_most_alternatives_of_the_longest_short_rows(V, K, dtype):
    """From 63 alternatives on, the room of a workgroup's four rows passes 64 KB of shared memory."""
    s = make(9, V, dtype, 14, "rows")
    check(s, run(s, 1.0, K, grad=False), 1.0, K)


def low_scores(V):
    """Rows that hold the type's lowest value, which a scale above one takes to -infinity."""
    s = make(4, V, "fp32", 15)
    low = torch.finfo(f32).min
    s["logits"][0] = low                                           # nothing has a probability
    s["logits"][1] = low
    s["logits"][1, V // 2] = 1.0                                   # one entry has
    s["token"][1] = V - 1                                          # and it is not the token
    s["logits"][2, ::2] = low
    s["token"][2] = 0
    return s


@pytest.mark.parametrize("V", [7, 40, 300, 900, 3000, 30000])
@pytest.mark.parametrize("gap", [0, 5])
def test_a_score_of_minus_infinity_has_no_probability_whatever_the_logit(V, gap):
    """Forward, alternatives and gradient agree that what counts is scale * logit."""
    K, scale = 4, 1.25
    s = low_scores(V)
    dead = s["logits"] == torch.finfo(f32).min
    if gap:                                                        # rows that are read one by one
        s["logits"] = torch.cat([s["logits"], torch.zeros(4, gap)], 1)
    o = run(s, scale, K)
    want = dict(s, logits=s["logits"].clone())
    want["logits"][:, :V][dead] = -float("inf")                    # the same rows without those entries
    check(want, o, scale, K)
    assert o["logp"][0] == 0 and o["logp"][1] == -float("inf") and o["logp"][2] == -float("inf")
    assert o["top_id"][0].eq(-1).all() and o["top_id"][1].tolist() == [V // 2, -1, -1, -1]
    assert (o["top_logp"][0] == -float("inf")).all() and not o["grad"].cpu()[dead].any()


@pytest.mark.parametrize("V", [7, 40, 300, 900, 3000, 30000])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("parts", [("logp",), ("entropy",), ("logp", "entropy")])
def test_the_gradient_of_a_row_that_is_not_finite_is_not_finite(V, value, parts):
    """NaN in every place that is available, so that a check of the gradients sees it; masked places stay 0."""
    for gap in (0, 5):
        s = make(3, V, "fp32", 16, "rows", V + gap, V + gap)
        s["avail"][1] = 1
        s["avail"][1, 2] = 0
        s["logits"][1] = 0.5
        clean = run(s, 1.0, 0, parts=parts)
        s["logits"][1, V - 2] = value
        o = run(s, 1.0, 0, parts=parts)
        here = s["avail"][1, :V] != 0
        assert torch.isnan(o["grad"][1].cpu()[here]).all() and not o["grad"][1, 2]
        assert torch.equal(o["grad"][::2], clean["grad"][::2])
