"""The gated linear recurrence on the GPU against the 64-bit oracle.

Tolerance.  A step's a and beta come out of a handful of fp32 operations, two to four half steps of 2^-24 each: below
2^-21 of the value.  The inputs' retention (0.9 .. 0.999 at an eighth of the gate) lets about 250 steps add up, so
a state is within 250 * 2^-21 = 1.2e-4 of the largest state, and so is every gradient of its own largest; the sum for
lam within that of the sum of its terms' sizes.  16-bit outputs add half a step of their own.
"""
import numpy as np
import pytest
import torch

from oracle import policy_oracle as orc
from policy_util import DT, gen, host, near, randn
from paper_2205_05248_amd import binding

pytestmark = pytest.mark.gpu
REL = 250 * 2.0 ** -21
DECAY = 8.0


def make(B, T, C, dtype, seed, reset=False, filled=False, first=True, layout="plain"):
    """CPU tensors; layout: "plain", "fused" (column blocks of one tensor), "shifted" (blocks at an odd element)."""
    g = gen(seed)
    dt = DT[dtype]
    s = dict(lam=torch.log(torch.expm1(-torch.log(0.9 + 0.099 * torch.rand(C, generator=g)))))
    s["xri"] = randn(g, B, T, 3, C, dtype=dt)
    s["reset"] = (torch.rand(B, T, generator=g) < 0.1).to(torch.uint8) if reset else None
    if filled:
        f = torch.rand(B, T, generator=g) < 0.8
        f[-1] = B == 1                                          # a row without a step, if there are several
        f[0, T // 2:] &= B > 2                                  # an early end
        s["filled"] = f.to(torch.uint8)
        s["xri"][~f] = float("nan")                             # what stands in padding does not matter
    else:
        s["filled"] = None
    s["h_first"] = randn(g, B, C) if first else None
    s["grad_y"] = randn(g, B, T, C, dtype=dt)
    if filled:
        s["grad_y"][~f] = float("inf")
    s["grad_h_last"] = randn(g, B, C) if first else None
    s["layout"] = layout
    return s


def on_gpu(s):
    B, T, _, C = s["xri"].shape
    xri = s["xri"].cuda()
    if s["layout"] == "plain":
        x, r, i = (xri[:, :, k].contiguous() for k in range(3))
    else:
        shift = 1 if s["layout"] == "shifted" else 0
        wide = torch.zeros(B, T, 3 * C + 2 * shift, dtype=xri.dtype, device="cuda")
        x, r, i = (wide[..., shift + k * C:shift + (k + 1) * C] for k in range(3))
        for k, t in enumerate((x, r, i)):
            t.copy_(xri[:, :, k])
    d = {k: (s[k].cuda() if torch.is_tensor(s[k]) else None) for k in ("lam", "reset", "filled", "h_first", "grad_y", "grad_h_last")}
    return dict(x=x, r=r, i=i, **d)


def outputs(d):
    B, T, C = d["x"].shape
    dt, nan = d["x"].dtype, float("nan")
    o = {k: torch.full((B, T, C), nan, dtype=dt, device="cuda") for k in ("y", "grad_x", "grad_r", "grad_i")}
    o.update(h_last=torch.full((B, C), nan, device="cuda"), grad_lam=torch.full((C,), nan, device="cuda"),
             grad_h_first=torch.full((B, C), nan, device="cuda"))
    name = {v: k for k, v in DT.items()}[dt]
    o["ws"] = torch.empty(binding.marl_linear_scan_workspace_bytes(name, B, T, C), dtype=torch.uint8, device="cuda").fill_(0xff)
    return o


def run(d, o):
    binding.marl_linear_scan(d["x"], d["r"], d["i"], d["lam"], DECAY, d["reset"], d["filled"], d["h_first"], o["y"], o["h_last"], o["ws"])
    binding.marl_linear_scan_grad(d["x"], d["r"], d["i"], d["lam"], DECAY, d["reset"], d["filled"], d["grad_y"], d["grad_h_last"], o["ws"],
                                  o["grad_x"], o["grad_r"], o["grad_i"], o["grad_lam"], o["grad_h_first"])


def check(s, o):
    x, r, i = (host(s["xri"][:, :, k]) for k in range(3))
    fill = host(s["filled"])
    clean = (lambda v: v) if fill is None else (lambda v: np.where(fill[..., None] != 0, v, 0.0))
    x, r, i, gy = clean(x), clean(r), clean(i), clean(host(s["grad_y"]))
    args = (x, r, i, host(s["lam"]), DECAY, host(s["reset"]), fill, host(s["h_first"]))
    y, last, _ = orc.linear_scan(*args)
    gx, gr, gi, glam, gh = orc.linear_scan_grad(*args, gy, host(s["grad_h_last"]))
    dt, f32 = s["xri"].dtype, torch.float32
    near(o["y"], y, dt, REL, "y")
    near(o["h_last"], last, f32, REL, "h_last")
    near(o["grad_x"], gx, dt, REL, "grad_x")
    near(o["grad_r"], gr, dt, REL, "grad_r")
    near(o["grad_i"], gi, dt, REL, "grad_i")
    near(o["grad_h_first"], gh, f32, REL, "grad_h_first")
    rate, by_lam = orc.rates(host(s["lam"]), DECAY)
    s_r = 1 / (1 + np.exp(-r))
    sizes = (np.abs(gr) / (rate * (1 - s_r))).sum((0, 1)) * by_lam
    near(o["grad_lam"], glam, f32, REL, "grad_lam", floor=sizes)


SIZES = [(1, 1, 1), (3, 2, 5), (2, 17, 33), (1, 127, 64), (1, 128, 8), (2, 129, 130), (4, 33, 512), (1, 1000, 40), (40, 12, 64), (1, 2055, 100)]


@pytest.mark.parametrize("B,T,C", SIZES)
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_forward_and_backward(B, T, C, dtype):
    k = SIZES.index((B, T, C))
    s = make(B, T, C, dtype, 10 + k, reset=k % 2 == 1, filled=k % 3 == 2, first=k % 4 != 3, layout=("plain", "fused", "shifted")[k % 3])
    d = on_gpu(s)
    o = outputs(d)
    run(d, o)
    torch.cuda.synchronize()
    check(s, o)


@pytest.mark.parametrize("reset,filled", [(False, False), (True, False), (False, True), (True, True)])
@pytest.mark.parametrize("layout", ["plain", "shifted"])
def test_masks_over_several_blocks(reset, filled, layout):
    s = make(3, 700, 72, "bf16", 77, reset, filled, True, layout)
    d = on_gpu(s)
    o = outputs(d)
    run(d, o)
    torch.cuda.synchronize()
    check(s, o)


def test_no_step_at_all():
    s = make(2, 0, 6, "fp32", 5)
    d = on_gpu(s)
    o = outputs(d)
    run(d, o)
    torch.cuda.synchronize()
    assert torch.equal(o["h_last"], d["h_first"]) and torch.equal(o["grad_h_first"], d["grad_h_last"]) and not o["grad_lam"].any()


def test_gates_at_their_ends():
    """Gates that are shut, open or far out: no infinity from 1 / beta, no NaN."""
    s = make(1, 40, 16, "fp32", 6)
    s["xri"][0, ::3, 1] = -200.0                                   # a = 1, beta = 0
    s["xri"][0, 1::3, 1] = 200.0
    s["xri"][0, 5, 2], s["xri"][0, 9, 2] = -200.0, 200.0
    s["lam"][3], s["lam"][4] = 60.0, -60.0
    d = on_gpu(s)
    o = outputs(d)
    run(d, o)
    torch.cuda.synchronize()
    x, r, i = (host(s["xri"][:, :, k]) for k in range(3))
    y, last, _ = orc.linear_scan(x, r, i, host(s["lam"]), DECAY, None, None, host(s["h_first"]))
    near(o["y"], y, torch.float32, REL, "y")
    near(o["h_last"], last, torch.float32, REL, "h_last")
    for k in ("grad_x", "grad_r", "grad_i", "grad_lam", "grad_h_first"):
        assert torch.isfinite(o[k]).all(), k


def test_outputs_as_column_blocks_and_states_in_place():
    s = make(2, 150, 24, "bf16", 8, reset=True)
    d = on_gpu(s)
    o = outputs(d)
    run(d, o)
    wide = torch.full((2, 150, 5 * 24), 7.0, dtype=torch.bfloat16, device="cuda")
    p = dict(o, y=wide[..., :24], grad_x=wide[..., 24:48], grad_r=wide[..., 48:72], grad_i=wide[..., 72:96], h_last=d["h_first"].clone(),
             grad_h_first=d["grad_h_last"].clone(), grad_lam=torch.empty_like(o["grad_lam"]))
    e = dict(d, h_first=p["h_last"], grad_h_last=p["grad_h_first"])
    run(e, p)
    torch.cuda.synchronize()
    for k in ("y", "grad_x", "grad_r", "grad_i", "h_last", "grad_lam", "grad_h_first"):
        assert torch.equal(o[k], p[k]), k
    assert (wide[..., 96:] == 7).all()


def test_same_bits_on_every_run_and_on_another_stream():
    s = make(1, 5000, 96, "fp32", 9, reset=True)
    d = on_gpu(s)
    first = outputs(d)
    run(d, first)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        o = outputs(d)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            run(d, o)
        side.synchronize()
        for k in first:
            if k != "ws":
                assert torch.equal(first[k], o[k]), k


def test_replayed_from_a_graph():
    s = make(2, 600, 128, "bf16", 11, reset=True, filled=True)
    d = on_gpu(s)
    d = {k: (None if v is None else v.clone()) for k, v in d.items()}
    o = outputs(d)
    run(d, o)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(d, o)
    for k in range(3):
        d["x"].mul_(0.5)
        want = outputs(d)
        run(d, want)
        for v in o:
            if v != "ws":
                o[v].zero_()
        graph.replay()
        torch.cuda.synchronize()
        for v in o:
            if v != "ws":
                assert torch.equal(o[v], want[v]), (k, v)


@pytest.mark.parametrize("n,C,slots,dtype", [(1, 1, 1, "fp32"), (24, 64, 24, "fp32"), (7, 33, 50, "bf16"), (130, 257, 200, "fp16"), (65, 2048, 65, "bf16")])
@pytest.mark.parametrize("listed", [True, False])
def test_single_steps(n, C, slots, dtype, listed):
    g = gen(n + C)
    s = make(1, n, C, dtype, n, layout="shifted" if C % 2 else "fused")
    d = {k: (v[0] if k in "xri" else v) for k, v in on_gpu(s).items()}
    slot = torch.randperm(slots, generator=g)[:n].to(torch.int32) if listed else None
    reset = (torch.rand(n, generator=g) < 0.3).to(torch.uint8) if n > 1 else None
    table = randn(g, slots, C)
    dev = table.cuda()
    y = torch.full((n, C), float("nan"), dtype=DT[dtype], device="cuda")
    binding.marl_linear_step(d["x"], d["r"], d["i"], d["lam"], DECAY, None if slot is None else slot.cuda(), None if reset is None else reset.cuda(),
                             dev, dev, y)
    torch.cuda.synchronize()
    x, r, i = (host(s["xri"][0, :, k]) for k in range(3))
    want, after = orc.linear_step(x, r, i, host(s["lam"]), DECAY, host(slot), host(reset), host(table))
    rel = 2.0 ** -20                                               # one step: a handful of operations
    near(y, want, DT[dtype], rel, "y")
    near(dev, after, torch.float32, rel, "h_out")
    rest = torch.ones(slots, dtype=torch.bool)
    rest[slot.long() if listed else torch.arange(n)] = False
    assert torch.equal(dev.cpu()[rest], table[rest])


def test_steps_follow_the_scan():
    s = make(3, 9, 40, "fp32", 12)
    d = on_gpu(s)
    o = outputs(d)
    run(d, o)
    h = d["h_first"].clone()
    for t in range(9):
        y = torch.empty(3, 40, device="cuda")
        binding.marl_linear_step(d["x"][:, t], d["r"][:, t], d["i"][:, t], d["lam"], DECAY, None, None, h, h, y)
        assert (y - o["y"][:, t]).abs().max() < REL
    assert (h - o["h_last"]).abs().max() < REL


def test_table_rows_out_of_range_are_clamped():
    s = make(1, 2, 8, "fp32", 13)
    d = {k: (v[0] if k in "xri" else v) for k, v in on_gpu(s).items()}
    table, y = torch.ones(4, 8, device="cuda"), torch.empty(2, 8, device="cuda")
    out = table.clone()
    binding.marl_linear_step(d["x"], d["r"], d["i"], d["lam"], DECAY, torch.tensor([-5, 99], dtype=torch.int32, device="cuda"), None, table, out, y)
    torch.cuda.synchronize()
    assert torch.equal(out[0], y[0]) and torch.equal(out[3], y[1]) and (out[1:3] == 1).all()


@pytest.mark.parametrize("T,C,dtype", [(30000, 64, "fp32"), (9000, 640, "bf16")])
def test_same_bits_beside_other_work(T, C, dtype):
    """When units begin and how long they take is not what decides about the order of a sum."""
    s = make(1, T, C, dtype, 20)
    d = on_gpu(s)
    first = outputs(d)
    run(d, first)
    torch.cuda.synchronize()
    side, big = torch.cuda.Stream(), torch.zeros(1 << 24, device="cuda")
    for n in range(6):
        o = outputs(d)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            for _ in range(2 * n):
                big.add_(1.0)
        run(d, o)
        torch.cuda.synchronize()
        for k in first:
            if k != "ws":
                assert torch.equal(first[k], o[k]), (n, k)


@pytest.mark.parametrize("B,T,C", [(2, 9, 3), (1, 90, 70), (2, 700, 66)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_a_reset_lets_nothing_through(B, T, C, dtype, value):
    """What a sequence holds, or its gradient, infinities and NaN too, reaches neither the next one nor the one before."""
    s = make(B, T, C, dtype, 21)
    cut = T // 3, 2 * T // 3                                       # three sequences a row; the middle one is spoiled
    s["reset"] = torch.zeros(B, T, dtype=torch.uint8)
    s["reset"][:, 0] = 1
    s["reset"][:, cut[0]], s["reset"][:, cut[1]] = 1, 1
    clean_in = on_gpu(s)
    clean = outputs(clean_in)
    run(clean_in, clean)
    at = (cut[0] + cut[1]) // 2
    s["xri"][0, at, 0, C // 2] = value
    s["xri"][0, cut[0] + 1, 1, C - 1] = float("nan")               # a gate: the decay itself is NaN
    s["grad_y"][0, at, 0] = value
    s["h_first"][0, C // 2] = value                                # a table's row that was never written
    d = on_gpu(s)
    o = outputs(d)
    run(d, o)
    torch.cuda.synchronize()
    for k in ("y", "grad_x", "grad_r", "grad_i"):
        for part in (slice(0, cut[0]), slice(cut[1], T)):
            assert torch.equal(o[k][:, part], clean[k][:, part]), (k, part)
    assert torch.equal(o["h_last"], clean["h_last"]) and torch.equal(o["grad_h_first"], clean["grad_h_first"])
    assert not torch.isfinite(o["y"][0, at, C // 2]) and torch.isnan(o["y"][0, at, C - 1])


def test_single_steps_of_more_rows_than_the_chip_holds_at_a_time():
    n, C = 600, 4096
    s = make(1, n, C, "bf16", 22, layout="fused")
    d = {k: (v[0] if k in "xri" else v) for k, v in on_gpu(s).items()}
    slot = torch.randperm(n + 50, generator=gen(22))[:n].to(torch.int32)
    table = randn(gen(23), n + 50, C)
    dev, y = table.cuda(), torch.empty(n, C, dtype=torch.bfloat16, device="cuda")
    binding.marl_linear_step(d["x"], d["r"], d["i"], d["lam"], DECAY, slot.cuda(), None, dev, dev, y)
    torch.cuda.synchronize()
    x, r, i = (host(s["xri"][0, :, k]) for k in range(3))
    want, after = orc.linear_step(x, r, i, host(s["lam"]), DECAY, host(slot), None, host(table))
    near(y, want, torch.bfloat16, 2.0 ** -20, "y")
    near(dev, after, torch.float32, 2.0 ** -20, "h_out")


def fast_channels(B, T, C, dtype, seed):
    """Channels whose decays' product over a stretch of steps is far below the smallest fp32 number, without any reset."""
    s = make(B, T, C, dtype, seed)
    s["lam"] = torch.full((C,), 3.0)                               # half a gate keeps e^-12 of the state
    s["lam"][C // 3] = 60.0                                        # and here nothing, to the last bit
    return s


def steps_from(s, value_of_h):
    """The states of the same sequences, step by step."""
    d = on_gpu(s)
    B, T, C = d["x"].shape
    h, states = value_of_h.clone(), []
    for t in range(T):
        y = torch.empty(B, C, dtype=d["x"].dtype, device="cuda")
        binding.marl_linear_step(d["x"][:, t], d["r"][:, t], d["i"][:, t], d["lam"], DECAY, None, None, h, h, y)
        states.append(h.clone())
    return torch.stack(states, 1)


@pytest.mark.parametrize("B,T,C", [(2, 9, 3), (1, 90, 70), (2, 700, 66)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("where", ["h_first", "x", "r"])
def test_what_is_not_finite_stays_until_a_reset(B, T, C, dtype, value, where):
    """However far the state decays: 0 times infinity or NaN is NaN, as step by step; and it stays in its channel and sequence."""
    if where == "r":
        value = float("nan")
    s = fast_channels(B, T, C, dtype, 24)
    clean_in = on_gpu(s)
    clean = outputs(clean_in)
    run(clean_in, clean)
    t0, channels = (0 if where == "h_first" else T // 4), sorted({0, C // 3, C - 1})
    for c in channels:
        if where == "h_first":
            s["h_first"][0, c] = value
        else:
            s["xri"][0, t0, "xri".index(where), c] = value
    d = on_gpu(s)
    o = outputs(d)
    run(d, o)
    torch.cuda.synchronize()
    spoiled = torch.zeros(B, T, C, dtype=torch.bool, device="cuda")
    spoiled[0, t0:, channels] = True
    assert not torch.isfinite(o["y"][spoiled]).any() and not torch.isfinite(o["h_last"][0, channels]).any()
    assert torch.equal(o["y"][~spoiled], clean["y"][~spoiled])
    assert torch.equal(torch.isfinite(steps_from(s, d["h_first"])[:, -1]), torch.isfinite(o["h_last"]))
    after = spoiled.clone()                                        # the gate's gradient has the state before the step as a factor
    if where != "h_first":
        after[0, t0] = False
    assert not torch.isfinite(o["grad_r"][after]).any()
    assert not torch.isfinite(o["grad_lam"][channels]).any()
    others = [c for c in range(C) if c not in channels]
    for k in ("grad_x", "grad_r", "grad_i"):
        assert torch.equal(o[k][..., others], clean[k][..., others]), k
    assert torch.equal(o["grad_lam"][others], clean["grad_lam"][others])


@pytest.mark.parametrize("B,T,C", [(2, 9, 3), (1, 90, 70), (2, 700, 66)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("where", ["grad_h_last", "grad_y"])
def test_a_gradient_that_is_not_finite_reaches_the_start(B, T, C, dtype, value, where):
    s = fast_channels(B, T, C, dtype, 25)
    clean_in = on_gpu(s)
    clean = outputs(clean_in)
    run(clean_in, clean)
    t1, channels = (T - 1 if where == "grad_h_last" else 3 * T // 4), sorted({0, C // 3, C - 1})
    for c in channels:
        if where == "grad_h_last":
            s["grad_h_last"][0, c] = value
        else:
            s["grad_y"][0, t1, c] = value
    d = on_gpu(s)
    o = outputs(d)
    run(d, o)
    torch.cuda.synchronize()
    spoiled = torch.zeros(B, T, C, dtype=torch.bool, device="cuda")
    spoiled[0, :t1 + 1, channels] = True
    for k in ("grad_x", "grad_r", "grad_i"):
        assert not torch.isfinite(o[k][spoiled]).any(), k
        assert torch.equal(o[k][~spoiled], clean[k][~spoiled]), k
    assert not torch.isfinite(o["grad_h_first"][0, channels]).any() and not torch.isfinite(o["grad_lam"][channels]).any()
    assert torch.equal(o["y"], clean["y"])


@pytest.mark.parametrize("B,T,C", [(2, 9, 3), (1, 90, 70), (2, 700, 66)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_a_nan_of_the_input_gate_is_in_its_gradients(B, T, C, dtype):
    s = make(B, T, C, dtype, 26)
    t0 = T // 2
    s["xri"][0, t0, 2, C - 1] = float("nan")
    d = on_gpu(s)
    o = outputs(d)
    run(d, o)
    torch.cuda.synchronize()
    for k in ("y", "grad_x", "grad_i"):
        assert torch.isnan(o[k][0, t0, C - 1]), k
    assert torch.isnan(o["grad_r"][0, t0:, C - 1]).all() and torch.isnan(o["grad_lam"][C - 1])


@pytest.mark.parametrize("B,T,C", [(2, 9, 3), (1, 90, 70), (2, 700, 66)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_the_gate_of_a_step_that_starts_a_sequence_is_not_looked_at(B, T, C, dtype, value):
    s = make(B, T, C, dtype, 27, reset=True, layout="shifted")
    s["reset"][:, T // 2] = 1
    start = s["reset"] != 0
    outs = []
    for v in (0.5, value):
        s["xri"][:, :, 1][start] = v
        d = on_gpu(s)
        outs.append(outputs(d))
        run(d, outs[-1])
    torch.cuda.synchronize()
    for k in outs[0]:
        if k != "ws":
            assert torch.equal(outs[0][k], outs[1][k]), k
    assert not outs[1]["grad_r"].cpu()[start].any()
    s["xri"][:, :, 1][start] = value
    check(dict(s, xri=torch.where(torch.isfinite(s["xri"]), s["xri"], torch.full_like(s["xri"], 0.5))), outs[1])


@pytest.mark.parametrize("C", [3, 64])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_the_gate_of_a_single_step_that_starts_a_sequence_is_not_looked_at(C, dtype, value):
    s = make(1, 5, C, dtype, 28)
    reset = torch.tensor([1, 0, 1, 0, 1], dtype=torch.uint8)
    ys = []
    for v in (0.5, value):
        s["xri"][0, reset != 0, 1] = v
        d = {k: (t[0].contiguous() if k in "xri" else t) for k, t in on_gpu(s).items()}
        table, y = torch.full((5, C), 2.0, device="cuda"), torch.empty(5, C, dtype=DT[dtype], device="cuda")
        table[0] = float("nan")
        binding.marl_linear_step(d["x"], d["r"], d["i"], d["lam"], DECAY, None, reset.cuda(), table, table, y)
        ys.append((y, table))
    torch.cuda.synchronize()
    assert torch.equal(ys[0][0], ys[1][0]) and torch.equal(ys[0][1], ys[1][1]) and torch.isfinite(ys[1][1]).all()


@pytest.mark.parametrize("T", [9, 90, 700])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_an_infinite_input_of_a_sequence_of_one_step_leaves_the_decay_alone(T, dtype):
    """grad_r of a step that starts a sequence is 0, and so is its part of grad_lam, whatever x is."""
    s = make(1, T, 5, dtype, 29)
    t0 = T // 2
    s["reset"] = torch.zeros(1, T, dtype=torch.uint8)
    s["reset"][:, t0:t0 + 2] = 1
    clean_in = on_gpu(s)
    clean = outputs(clean_in)
    run(clean_in, clean)
    s["xri"][0, t0, 0, 2] = float("inf")
    d = on_gpu(s)
    o = outputs(d)
    run(d, o)
    torch.cuda.synchronize()
    for k in ("grad_r", "grad_lam", "grad_h_first", "grad_x", "h_last"):
        assert torch.equal(o[k], clean[k]), k
    assert not o["grad_r"][0, t0:t0 + 2].any() and torch.isinf(o["y"][0, t0, 2])


@pytest.mark.parametrize("B,T,C", [(2, 9, 3), (2, 90, 70), (2, 700, 66)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_padding_has_no_gradient_whatever_passes_through_it(B, T, C, dtype, value):
    """A sequence without a step hands on what it is given, and adds nothing to grad_lam."""
    s = make(B, T, C, dtype, 30, filled=True)
    s["filled"][0] = 1
    s["filled"][0, T // 3:T // 2] = 0
    pad = s["filled"] == 0
    s["xri"][~pad] = randn(gen(31), int((~pad).sum()), 3, C, dtype=DT[dtype])
    s["grad_y"][~pad] = 1.0
    clean_in = on_gpu(s)
    clean = outputs(clean_in)
    run(clean_in, clean)
    s["h_first"][1, 0], s["grad_h_last"][1, C - 1] = value, value  # the row that is padding alone
    s["grad_y"][0, T // 2, C - 1] = value                          # and what passes the padding inside a row
    d = on_gpu(s)
    o = outputs(d)
    run(d, o)
    torch.cuda.synchronize()
    for k in ("y", "grad_x", "grad_r", "grad_i"):
        assert not o[k].cpu()[pad].any(), k                        # (NaN counts as something)
    assert torch.equal(o["grad_lam"][:C - 1], clean["grad_lam"][:C - 1])
    assert not torch.isfinite(o["h_last"][1, 0]) and not torch.isfinite(o["grad_h_first"][1, C - 1])


@pytest.mark.parametrize("T", [5, 60, 300])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_gradient_of_gates_that_are_almost_open_or_shut(T, dtype):
    """Entry by entry: sigmoid(r) (1 - sigmoid(r)) keeps its digits at both ends.  The other factors of grad_r are within REL of their
    largest values, and so is the product of the sizes (three factors of a few operations more)."""
    C = 40
    s = make(1, T, C, dtype, 32)
    s["xri"][0, :, 1] = torch.linspace(-20, 20, T * C).view(C, T).t().to(DT[dtype])
    s["lam"] = torch.linspace(-4, -1, C)
    d = on_gpu(s)
    o = outputs(d)
    run(d, o)
    torch.cuda.synchronize()
    x, r, i = (host(s["xri"][:, :, k]) for k in range(3))
    args = (x, r, i, host(s["lam"]), DECAY, None, None, host(s["h_first"]))
    _, _, before = orc.linear_scan(*args)
    want = orc.linear_scan_grad(*args, host(s["grad_y"]), host(s["grad_h_last"]))[1]
    rate, _ = orc.rates(host(s["lam"]), DECAY)
    e = np.exp(-np.abs(r))
    s_r, slope = np.where(r > 0, 1 / (1 + e), e / (1 + e)), e / (1 + e) ** 2
    a, beta = np.exp(-rate * s_r), np.sqrt(-np.expm1(-2 * rate * s_r))
    q0 = np.abs(x) / (1 + np.exp(-i)) * a / beta
    dh = adjoint(a, host(s["grad_y"]), host(s["grad_h_last"]))
    sizes = rate * slope * (a * np.abs(dh).max() * (np.abs(before).max() + q0))
    near(o["grad_r"], want, DT[dtype], 2 * REL, "grad_r", floor=sizes)


def adjoint(a, grad_y, grad_h_last):
    """dL/dh of every step."""
    dh, out = grad_h_last, np.zeros(a.shape)
    for t in range(a.shape[1] - 1, -1, -1):
        out[:, t] = dh + grad_y[:, t]
        dh = a[:, t] * out[:, t]
    return out
