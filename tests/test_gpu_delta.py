"""Gated delta rule on the GPU against the 64-bit oracle: sequences there and back, single steps, masks, strides, what is not finite.

Tolerance.  Inputs of the oracle are the rounded ones the kernels get.  Within a chunk of 64 steps a value passes four products one after the
other (with the state, with N, with P, into the state), sums of at most 128, 64, 64 and 64 terms, each term and each addition rounded to
2^-24 of what it is: 320 roundings, and as many again for the factors that the terms carry (decays, beta, N itself).  All in the same direction
they would add up to 640 x 2^-24 of the sum of the terms' sizes; the inputs here have random signs, for which the sum of sizes is at
most sqrt(128) of the result's own scale and the roundings add up like a random walk, sqrt(640) x 2^-24 x sqrt(128) = 1.7e-5 = 2^-15.8 of the
scale.  Backward the sums are twice as long.  So: 2^-15 of the largest value for any single one, on top of half a step of the
result's type; and over all of a result, where single large deviations average out, 2^-18 of its norm.
"""
import numpy as np
import pytest
import torch

from oracle import memory_oracle as orc
from paper_2205_05248_amd import binding
from policy_util import DT, gen, host, near, randn

pytestmark = pytest.mark.gpu
REL, NORM = 2.0 ** -15, 2.0 ** -18
f32 = torch.float32


def make(B, T, Hk, Hv, Dk, Dv, dtype, seed, reset=None, filled=None, first=True, gap=0):
    """Tensors on the host; `gap` unused elements behind every row."""
    g = gen(seed)
    unit = lambda t: t / t.norm(dim=-1, keepdim=True).clamp(min=1e-3)
    wide = lambda t: torch.cat([t.flatten(2), torch.full((B, T, gap), float("nan"))], 2)[..., :t.shape[2] * t.shape[3]].unflatten(2, t.shape[2:]) if gap else t
    s = dict(q=wide(unit(randn(g, B, T, Hk, Dk)).to(DT[dtype]).float()).to(DT[dtype]), k=unit(randn(g, B, T, Hk, Dk)).to(DT[dtype]),
             v=randn(g, B, T, Hv, Dv).to(DT[dtype]), log_decay=-0.3 * torch.rand(B, T, Hv, generator=g), beta=torch.rand(B, T, Hv, generator=g),
             scale=Dk ** -0.5, s_first=randn(g, B, Hv, Dk, Dv) * 0.5 if first else None, reset=reset, filled=filled,
             grad_o=randn(g, B, T, Hv, Dv).to(DT[dtype]), grad_s_last=randn(g, B, Hv, Dk, Dv) * 0.5)
    return s


def cuda(t, gap=0):
    """On the device; with a gap, rows lie in a wider array whose rest is NaN."""
    if t is None or not gap or t.dim() < 3:
        return None if t is None else t.cuda()
    lead = t.shape[:-2]
    H, D = t.shape[-2:]
    wide = torch.full((*lead, H * D + gap), float("nan"), dtype=t.dtype, device="cuda")
    wide[..., :H * D] = t.flatten(-2).cuda()
    return wide[..., :H * D].unflatten(-1, (H, D))


def run(s, train=True, gap=0, last=True):
    B, T, Hk, Dk = s["q"].shape
    Hv, Dv = s["v"].shape[2:]
    dt = s["q"].dtype
    name = {v: k for k, v in DT.items()}[dt]
    d = {k: cuda(v, gap if k in ("q", "k", "v", "grad_o") else 0) if torch.is_tensor(v) else v for k, v in s.items()}
    nan = lambda *shape, dtype=f32: torch.full(shape, float("nan"), dtype=dtype, device="cuda")
    o = dict(o=cuda(nan(B, T, Hv, Dv, dtype=dt), gap), s_last=nan(B, Hv, Dk, Dv) if last else None)
    ws = torch.empty(binding.marl_delta_scan_workspace_bytes(name, B, T, Hk, Hv, Dk, Dv, train), dtype=torch.uint8, device="cuda").fill_(0xff)
    binding.marl_delta_scan(d["q"], d["k"], d["v"], d["log_decay"], d["beta"], s["scale"], d["reset"], d["filled"], d["s_first"], o["o"], o["s_last"],
                            ws, keep=train)
    if train:
        o.update(grad_q=cuda(nan(B, T, Hk, Dk, dtype=dt), gap), grad_k=cuda(nan(B, T, Hk, Dk, dtype=dt), gap), grad_v=cuda(nan(B, T, Hv, Dv, dtype=dt), gap),
                 grad_log_decay=nan(B, T, Hv), grad_beta=nan(B, T, Hv), grad_s_first=nan(B, Hv, Dk, Dv))
        binding.marl_delta_scan_grad(d["q"], d["k"], d["v"], d["log_decay"], d["beta"], s["scale"], d["reset"], d["filled"], d["grad_o"],
                                     d["grad_s_last"], ws, o["grad_q"], o["grad_k"], o["grad_v"], o["grad_log_decay"], o["grad_beta"], o["grad_s_first"])
    torch.cuda.synchronize()
    return o


def wanted(s, train=True):
    a = {k: host(v) if torch.is_tensor(v) else v for k, v in s.items()}
    want = {}
    want["o"], want["s_last"], _ = orc.delta_scan(a["q"], a["k"], a["v"], a["log_decay"], a["beta"], s["scale"], a["reset"], a["filled"], a["s_first"])
    if train:
        names = ("grad_q", "grad_k", "grad_v", "grad_log_decay", "grad_beta", "grad_s_first")
        want.update(zip(names, orc.delta_scan_grad(a["q"], a["k"], a["v"], a["log_decay"], a["beta"], s["scale"], a["reset"], a["filled"], a["s_first"],
                                                   a["grad_o"], a["grad_s_last"])))
    return want


def check(o, want):
    for name, w in want.items():
        if o.get(name) is None:
            continue
        dt = o[name].dtype
        near(o[name], w, dt, REL, name)
        if dt == f32 and w.size and np.isfinite(w).all():
            assert np.linalg.norm(host(o[name]) - w) <= NORM * np.linalg.norm(w) + 1e-30, name


SIZES = [(1, 1, 1, 1, 1, 1), (2, 5, 1, 2, 3, 2), (3, 64, 2, 2, 16, 16), (1, 65, 1, 1, 32, 33), (2, 130, 2, 4, 40, 72), (1, 200, 1, 3, 128, 128),
         (2, 63, 3, 3, 64, 17), (1, 129, 1, 1, 100, 200), (1, 257, 2, 2, 65, 16), (5, 16, 1, 8, 24, 8)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("size", SIZES)
def test_scan_there_and_back(size, dtype):
    s = make(*size, dtype, seed=sum(size))
    check(run(s), wanted(s))


def masks(B, T, seed, resets=0.1, lengths=True):
    r = np.random.default_rng(seed)
    reset = torch.from_numpy((r.random((B, T)) < resets).astype(np.uint8))
    length = r.integers(0, T + 1, B)
    length[0] = 0
    filled = torch.from_numpy((np.arange(T)[None] < length[:, None]).astype(np.uint8)) if lengths else torch.from_numpy((r.random((B, T)) < 0.7).astype(np.uint8))
    return reset, filled


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("resets,lengths", [(0.02, True), (0.5, True), (1.0, False), (0.05, False)])
def test_sequences_that_start_and_end(resets, lengths, dtype):
    """Padding may hold anything, its upstream gradient too."""
    B, T = 4, 150
    reset, filled = masks(B, T, 3, resets, lengths)
    s = make(B, T, 2, 4, 24, 20, dtype, 5, reset, filled)
    pad = filled == 0
    for name in ("q", "k", "v", "grad_o"):
        s[name][pad] = float("nan")
    s["log_decay"][pad] = float("inf")
    s["beta"][pad] = float("nan")
    clean = {**s, **{n: torch.nan_to_num(s[n], 0.0, 0.0, 0.0) for n in ("q", "k", "v", "grad_o", "log_decay", "beta")}}
    check(run(s), wanted(clean))


def test_decays_at_their_ends():
    """No decay at all, decays that leave nothing, -infinity (which forgets like a reset), -0."""
    s = make(2, 140, 1, 2, 16, 16, "fp32", 9)
    s["log_decay"][0] = 0.0
    s["log_decay"][1, ::7] = -float("inf")
    s["log_decay"][1, 3::11] = -1e30
    s["log_decay"][1, 5::13] = -120.0
    check(run(s), wanted(s))


def test_beta_of_zero_one_and_two():
    s = make(1, 100, 1, 3, 16, 16, "fp32", 11)
    s["beta"][0, :, 0], s["beta"][0, :, 1], s["beta"][0, ::2, 2] = 0.0, 1.0, 2.0
    s["log_decay"][0, :, 2] = -0.5
    check(run(s), wanted(s))


def test_keys_that_repeat():
    """The same key again and again, with beta 1 and little decay: every entry of A is next to 1."""
    s = make(1, 150, 1, 1, 8, 16, "fp32", 12)
    s["k"] = s["k"][:, :1].expand(-1, 150, -1, -1).contiguous()
    s["beta"][:] = 1.0
    s["log_decay"][:] = -1e-3
    check(run(s), wanted(s))


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_rows_of_wider_arrays(dtype):
    s = make(2, 70, 2, 2, 12, 20, dtype, 13)
    check(run(s, gap=5), wanted(s))


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("Dv,gap", [(17, 0), (17, 5), (31, 0), (32, 1), (33, 2), (50, 3)])
def test_two_columns_a_lane(Dv, gap, dtype):
    """Heads enough for the whole chip: a lane has two value columns, the last of an odd number one; rows begin at odd elements too."""
    for Dk, B in ((12, 64), (40, 64), (70, 32)):
        s = make(B, 66, 2, 8, Dk, Dv, dtype, 70 + Dv, *masks(B, 66, Dv, 0.05))
        check(run(s, gap=gap), wanted(s))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("size", [(2, 70, 1, 9, 20, 12), (1, 65, 2, 10, 128, 40), (1, 130, 1, 5, 64, 90)])
def test_many_heads_of_one_key(size, dtype):
    s = make(*size, dtype, 80 + size[3], *masks(size[0], size[1], 9, 0.05, False))
    check(run(s), wanted(s))


def test_sequences_that_end_with_a_chunk():
    for T in (63, 64, 65, 128):
        s = make(3, T, 1, 2, 32, 32, "bf16", 90 + T)
        s["reset"] = torch.zeros(3, T, dtype=torch.uint8)
        s["reset"][0, -1], s["reset"][1, min(T - 1, 63)], s["reset"][2, min(T - 1, 64)] = 1, 1, 1
        check(run(s), wanted(s))


def test_forward_alone_and_without_states():
    s = make(2, 90, 1, 2, 16, 24, "bf16", 14, first=False)
    o = run(s, train=False, last=False)
    near(o["o"], wanted(s, False)["o"], torch.bfloat16, REL, "o")


def test_nothing_to_do():
    """T = 0 hands the state, and backward its gradient, through; B = 0 is no call."""
    s = make(2, 0, 1, 2, 4, 6, "fp32", 15)
    o = run(s)
    assert torch.equal(o["s_last"].cpu(), s["s_first"]) and torch.equal(o["grad_s_first"].cpu(), s["grad_s_last"])
    run(make(0, 5, 1, 2, 4, 6, "fp32", 16))


def test_state_in_place():
    s = make(2, 80, 1, 2, 16, 16, "fp32", 17)
    want = wanted(s, False)
    state = s["s_first"].cuda()
    o = torch.empty(2, 80, 2, 16, device="cuda")
    ws = torch.empty(binding.marl_delta_scan_workspace_bytes("fp32", 2, 80, 1, 2, 16, 16), dtype=torch.uint8, device="cuda")
    binding.marl_delta_scan(s["q"].cuda(), s["k"].cuda(), s["v"].cuda(), s["log_decay"].cuda(), s["beta"].cuda(), s["scale"], None, None, state, o, state, ws)
    check(dict(o=o, s_last=state), want)


@pytest.mark.parametrize("what", ["v", "k", "q", "beta", "s_first", "log_decay"])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_what_is_not_finite_stays_in_its_sequence(what, value):
    """Forward: no step before it, no other sequence and no other head is touched; where the recurrence gives a finite value, so do the kernels.
    Backward: no other sequence."""
    B, T, H = 2, 150, 2
    reset = torch.zeros(B, T, dtype=torch.uint8)
    reset[0, 20] = reset[0, 45] = reset[0, 100] = 1
    s = make(B, T, 1, H, 8, 16, "fp32", 18, reset=reset)
    if what == "s_first":
        s["s_first"][0, 1, 2, 3] = value
    elif what in ("q", "k"):
        s[what][0, 30, 0, 2] = value
    elif what == "v":
        s[what][0, 30, 1, 3] = value
    else:
        s[what][0, 30, 1] = value
    o = run(s)
    with np.errstate(invalid="ignore", over="ignore"):
        want = wanted(s)
    lo, hi = (0, 20) if what == "s_first" else (20, 45)
    got, w = host(o["o"]), want["o"]
    assert np.array_equal(np.isfinite(got), np.isfinite(w))
    ok = np.isfinite(w)
    assert np.abs(got - w)[ok].max() <= REL * np.abs(w[ok]).max()
    for name in ("grad_q", "grad_k", "grad_v", "grad_log_decay", "grad_beta"):
        g, w = host(o[name]), want[name]
        outside = np.ones((B, T), bool)
        outside[0, lo:hi] = False
        assert np.isfinite(w[outside]).all()
        assert np.abs(g[outside] - w[outside]).max() <= REL * np.abs(w[outside]).max(), name
    assert np.array_equal(np.isfinite(host(o["s_last"])), np.isfinite(want["s_last"]))


@pytest.mark.parametrize("what", ["grad_o", "grad_s_last"])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), torch.finfo(f32).max])
def test_an_upstream_gradient_that_is_not_finite_stays_in_its_sequence(what, value):
    B, T, H = 2, 150, 2
    reset = torch.zeros(B, T, dtype=torch.uint8)
    reset[0, 20] = reset[0, 45] = reset[0, 100] = 1
    s = make(B, T, 1, H, 8, 16, "fp32", 21, reset=reset)
    s[what][(0, 30, 1, 3) if what == "grad_o" else (0, 1, 2, 3)] = value
    o = run(s)
    with np.errstate(invalid="ignore", over="ignore"):
        want = wanted(s)
    outside = np.ones((B, T), bool)
    outside[0, slice(20, 45) if what == "grad_o" else slice(100, T)] = False
    for name in ("grad_q", "grad_k", "grad_v", "grad_log_decay", "grad_beta"):
        g, w = host(o[name])[outside], want[name][outside]
        assert np.abs(g - w).max() <= REL * np.abs(w).max(), name
    near(o["grad_s_first"], want["grad_s_first"], f32, REL, "grad_s_first")


@pytest.mark.parametrize("what", ["v", "k", "q", "s_first"])
def test_the_largest_numbers_stay_in_their_sequence(what):
    """As what is not finite, although they are."""
    B, T, H = 2, 150, 2
    reset = torch.zeros(B, T, dtype=torch.uint8)
    reset[0, 20] = reset[0, 45] = reset[0, 100] = 1
    s = make(B, T, 1, H, 8, 16, "fp32", 20, reset=reset)
    largest = torch.finfo(f32).max
    if what == "s_first":
        s["s_first"][0, 1, 2, 3] = -largest
    elif what == "v":
        s["v"][0, 30, 1, 3] = -largest
    else:
        s[what][0, 30, 0, 2] = largest
    o = run(s)
    with np.errstate(invalid="ignore", over="ignore"):
        want = wanted(s)
    lo, at, hi = (0, 0, 20) if what == "s_first" else (20, 30, 45)
    for name in ("o", "grad_q", "grad_k", "grad_v", "grad_log_decay", "grad_beta"):
        outside = np.ones((B, T), bool)
        outside[0, at if name == "o" else lo:hi] = False
        g, w = host(o[name])[outside], want[name][outside]
        assert np.abs(g - w).max() <= REL * np.abs(w).max(), name


def test_the_same_bits_again():
    reset, filled = masks(3, 200, 4)
    s = make(3, 200, 2, 4, 32, 48, "bf16", 19, reset, filled)
    a, b = run(s), run(s)
    for name in a:
        assert torch.equal(a[name], b[name]), name


def test_gradient_by_differences():
    """The kernels' own forward pass in fp32, differences of a loss along random directions, steps of 2^-7: the second-order part is below
    2^-14 of the loss's scale, its rounding 2^-17 x 2^7."""
    s = make(1, 70, 1, 2, 8, 8, "fp32", 20)
    o = run(s)
    go, gs = s["grad_o"].double(), s["grad_s_last"].double()

    def loss(d):
        r = run(d, train=False)
        return float((r["o"].double().cpu() * go).sum() + (r["s_last"].double().cpu() * gs).sum())

    g = gen(21)
    for name, grad in (("q", "grad_q"), ("k", "grad_k"), ("v", "grad_v"), ("log_decay", "grad_log_decay"), ("beta", "grad_beta"), ("s_first", "grad_s_first")):
        way = randn(g, *s[name].shape)
        way = way / way.norm()
        step = 2.0 ** -7
        diff = (loss({**s, name: s[name] + step * way}) - loss({**s, name: s[name] - step * way})) / (2 * step)
        along = float((o[grad].double().cpu() * way.double()).sum())
        scale = float(o[grad].double().norm()) + abs(loss(s)) * 2.0 ** -7
        assert abs(diff - along) <= 2.0 ** -8 * scale, (name, diff, along)


# ------------------------------------------------------------------------------------------------ single steps
def make_step(n, slots, Hk, Hv, Dk, Dv, dtype, seed, reset=False, slot=True):
    g = gen(seed)
    one = make(n, 1, Hk, Hv, Dk, Dv, dtype, seed)
    s = {k: one[k][:, 0] for k in ("q", "k", "v", "log_decay", "beta")}
    s.update(scale=one["scale"], s_in=randn(g, slots, Hv, Dk, Dv), slot=torch.randperm(slots, generator=g)[:n].to(torch.int32) if slot else None,
             reset=(torch.rand(n, generator=g) < 0.4).to(torch.uint8) if reset else None)
    return s


def run_step(s, gap=0, in_place=False):
    d = {k: cuda(v, gap if k in "qkv" else 0) if torch.is_tensor(v) else v for k, v in s.items()}
    out = d["s_in"] if in_place else torch.full_like(d["s_in"], 7.0)
    o = cuda(torch.full_like(s["v"], float("nan")), gap)
    binding.marl_delta_step(d["q"], d["k"], d["v"], d["log_decay"], d["beta"], s["scale"], d["slot"], d["reset"], d["s_in"], out, o)
    torch.cuda.synchronize()
    return o, out


STEPS = [(1, 1, 1, 1, 1, 1), (24, 24, 2, 2, 32, 32), (5, 9, 1, 3, 7, 10), (3, 4, 2, 4, 128, 128), (2, 3, 1, 1, 128, 1024), (4, 6, 1, 1, 33, 133), (6, 6, 1, 2, 64, 3)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("size", STEPS)
def test_step(size, dtype):
    s = make_step(*size, dtype, sum(size), reset=size[0] > 2)
    o, table = run_step(s, gap=3)
    a = {k: host(v) if torch.is_tensor(v) else v for k, v in s.items()}
    want_o, want = orc.delta_step(a["q"], a["k"], a["v"], a["log_decay"], a["beta"], s["scale"], a["slot"], a["reset"], a["s_in"])
    near(o, want_o, o.dtype, REL, "o")
    listed = a["slot"]
    near(table[listed.tolist()], want[listed], f32, REL, "table")
    others = np.setdiff1d(np.arange(size[1]), listed)
    assert (host(table)[others] == 7.0).all()


def test_step_in_place_and_without_slots():
    s = make_step(5, 8, 1, 2, 16, 20, "bf16", 30, slot=False)
    o, table = run_step(s, in_place=True)
    a = {k: host(v) if torch.is_tensor(v) else v for k, v in s.items()}
    want_o, want = orc.delta_step(a["q"], a["k"], a["v"], a["log_decay"], a["beta"], s["scale"], None, None, a["s_in"])
    near(o, want_o, o.dtype, REL, "o")
    near(table, want, f32, REL, "table")


def test_rows_of_a_table_behind_32_bits():
    """Entries behind 2^32 of a table, and rows of v and o as far apart as they may be."""
    slots = (1 << 32) // (128 * 128) + 5
    table = torch.empty(slots, 1, 128, 128, device="cuda")
    s = make_step(3, 4, 1, 1, 128, 128, "bf16", 33)
    s["slot"] = torch.tensor([0, 1, 3], dtype=torch.int32)
    where = torch.tensor([slots - 1, 7, slots - 4], dtype=torch.int32)
    others = torch.tensor([slots - 2, slots - 3, (slots - 1) % (1 << 18), 6, 8])
    table[others.cuda()] = 7.0
    table[where.long().cuda()] = s["s_in"][[0, 1, 3]].cuda()
    o = torch.empty(3, 1, 128, dtype=torch.bfloat16, device="cuda")
    d = [s[n].cuda() for n in ("q", "k", "v", "log_decay", "beta")]
    binding.marl_delta_step(*d, s["scale"], where.cuda(), None, table, table, o)
    a = {k: host(v) if torch.is_tensor(v) else v for k, v in s.items()}
    want_o, want = orc.delta_step(a["q"], a["k"], a["v"], a["log_decay"], a["beta"], s["scale"], a["slot"], None, a["s_in"])
    near(o, want_o, o.dtype, REL, "o")
    near(table[where.long().cuda()], want[[0, 1, 3]], f32, REL, "table")
    assert (table[others.cuda()] == 7.0).all()


def test_rows_as_far_apart_as_they_may_be():
    T, ld = 300, (1 << 24) - 1
    s = make(1, T, 1, 1, 16, 20, "bf16", 34)
    far = torch.empty(T * ld, dtype=torch.bfloat16, device="cuda")
    rows = lambda first, n: far[first:].as_strided((1, T, 1, n), (T * ld, ld, n, 1))
    v, o, grad_o, grad_v = rows(0, 20), rows(101, 20), rows(202, 20), rows(303, 20)
    q, k, grad_q, grad_k = rows(404, 16), rows(505, 16), rows(606, 16), rows(707, 16)
    for to, n in ((v, "v"), (grad_o, "grad_o"), (q, "q"), (k, "k")):
        to.copy_(s[n])
    d = {n: t.cuda() for n, t in s.items() if torch.is_tensor(t)}
    out = dict(o=o, s_last=torch.empty_like(d["s_first"]), grad_q=grad_q, grad_k=grad_k, grad_v=grad_v, grad_log_decay=torch.empty(1, T, 1, device="cuda"),
               grad_beta=torch.empty(1, T, 1, device="cuda"), grad_s_first=torch.empty_like(d["s_first"]))
    ws = torch.empty(binding.marl_delta_scan_workspace_bytes("bf16", 1, T, 1, 1, 16, 20, True), dtype=torch.uint8, device="cuda")
    binding.marl_delta_scan(q, k, v, d["log_decay"], d["beta"], s["scale"], None, None, d["s_first"], o, out["s_last"], ws, keep=True)
    binding.marl_delta_scan_grad(q, k, v, d["log_decay"], d["beta"], s["scale"], None, None, grad_o, d["grad_s_last"], ws, grad_q, grad_k, grad_v,
                                 out["grad_log_decay"], out["grad_beta"], out["grad_s_first"])
    check(out, wanted(s))


def test_step_forgets_what_is_not_finite():
    s = make_step(4, 4, 1, 1, 8, 8, "fp32", 31)
    s["reset"] = torch.tensor([1, 0, 0, 0], dtype=torch.uint8)
    s["log_decay"][1] = -float("inf")
    s["s_in"][s["slot"][0].item()] = float("nan")
    s["s_in"][s["slot"][1].item()] = float("inf")
    o, table = run_step(s)
    a = {k: host(v) if torch.is_tensor(v) else v for k, v in s.items()}
    want_o, want = orc.delta_step(a["q"], a["k"], a["v"], a["log_decay"], a["beta"], s["scale"], a["slot"], a["reset"], a["s_in"])
    near(o, want_o, f32, REL, "o")
    near(table[a["slot"].tolist()], want[a["slot"]], f32, REL, "table")


def test_steps_follow_the_scan():
    """One step after the other gives what the whole sequence gives."""
    s = make(3, 20, 1, 2, 16, 24, "fp32", 32)
    o = run(s, train=False)
    table, outs = s["s_first"].cuda(), []
    for t in range(20):
        out = torch.empty(3, 2, 24, device="cuda")
        args = [s[n][:, t].contiguous().cuda() for n in ("q", "k", "v", "log_decay", "beta")]
        binding.marl_delta_step(*args, s["scale"], None, None, table, table, out)
        outs.append(out)
    near(torch.stack(outs, 1), host(o["o"]), f32, REL, "o")
    near(table, host(o["s_last"]), f32, REL, "state")


# ------------------------------------------------------------------------------------------------ streams and graphs
def test_graph_of_scan_and_gradient():
    """Captured after an eager call, replayed with other inputs and eager work in between; every replay against the eager bits."""
    sets = [make(2, 100, 1, 2, 32, 32, "bf16", 40 + i) for i in range(3)]
    eager = [run(s) for s in sets]
    B, T, Hk, Hv, Dk, Dv = 2, 100, 1, 2, 32, 32
    names = ("q", "k", "v", "log_decay", "beta", "s_first", "grad_o", "grad_s_last")
    d = {n: sets[0][n].cuda().clone() for n in names}
    out = {n: torch.zeros_like(t) for n, t in eager[0].items()}
    ws = torch.empty(binding.marl_delta_scan_workspace_bytes("bf16", B, T, Hk, Hv, Dk, Dv, True), dtype=torch.uint8, device="cuda")

    def once():
        binding.marl_delta_scan(d["q"], d["k"], d["v"], d["log_decay"], d["beta"], sets[0]["scale"], None, None, d["s_first"], out["o"], out["s_last"], ws, keep=True)
        binding.marl_delta_scan_grad(d["q"], d["k"], d["v"], d["log_decay"], d["beta"], sets[0]["scale"], None, None, d["grad_o"], d["grad_s_last"], ws,
                                     out["grad_q"], out["grad_k"], out["grad_v"], out["grad_log_decay"], out["grad_beta"], out["grad_s_first"])

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        once()
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        once()
    for i in (1, 2, 0, 1):
        for n in names:
            d[n].copy_(sets[i][n])
        graph.replay()
        torch.cuda.synchronize()
        for n, t in eager[i].items():
            assert torch.equal(out[n], t), (i, n)
        run(sets[i])


def test_two_streams_side_by_side():
    a, b = make(4, 300, 1, 2, 64, 64, "bf16", 50), make(4, 300, 1, 2, 64, 64, "bf16", 51)
    alone = [run(a), run(b)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [None, None]
    torch.cuda.synchronize()
    for i, s in enumerate((a, b)):
        with torch.cuda.stream(streams[i]):
            outs[i] = run(s)
    torch.cuda.synchronize()
    for x, y in zip(alone, outs):
        for n in x:
            assert torch.equal(x[n], y[n]), n


def test_refused_tensors():
    s = make(2, 5, 1, 2, 4, 6, "fp32", 60)
    d = {k: v.cuda() if torch.is_tensor(v) else v for k, v in s.items()}
    o, ws = torch.empty(2, 5, 2, 6, device="cuda"), torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    call = lambda **k: binding.marl_delta_scan(*({**dict(q=d["q"], k=d["k"], v=d["v"], g=d["log_decay"], b=d["beta"], scale=0.5, reset=None, filled=None,
                                                          s=None, o=o, last=None, ws=ws), **k}).values())
    call()
    for bad in (dict(k=d["k"].half()), dict(q=s["q"]), dict(g=d["log_decay"][:, :4]), dict(o=o.transpose(0, 1)), dict(s=d["s_first"].half()),
                dict(v=torch.empty(2, 5, 6, 2, device="cuda").transpose(2, 3)), dict(reset=torch.zeros(2, 5, device="cuda"))):
        with pytest.raises(ValueError):
            call(**bad)
    with pytest.raises(binding.MarlError):
        call(ws=ws[:256])
