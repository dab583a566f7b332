"""The oracle of the delta rule, the distillation and the penalties against differences and small cases worked out by hand; and what the
entry points refuse before they touch a device."""
import ctypes

import numpy as np
import pytest

from oracle import memory_oracle as orc
from oracle import policy_oracle
from paper_2205_05248_amd import binding


def _delta(seed, B=2, T=5, Hk=2, Hv=4, Dk=3, Dv=2):
    r = np.random.default_rng(seed)
    s = dict(q=r.normal(size=(B, T, Hk, Dk)), k=r.normal(size=(B, T, Hk, Dk)) * 0.5, v=r.normal(size=(B, T, Hv, Dv)),
             log_decay=-r.random((B, T, Hv)), beta=r.random((B, T, Hv)), s_first=r.normal(size=(B, Hv, Dk, Dv)))
    reset, filled = np.zeros((B, T), np.uint8), np.ones((B, T), np.uint8)
    reset[0, 2:3] = 1
    filled[1, 3:] = 0
    return s, reset, filled


def test_delta_rule_writes_and_reads_back():
    """A unit key with beta 1 and no decay: the value under the key is replaced, and read back whole."""
    k = np.array([[[[1.0, 0.0]], [[0.0, 1.0]], [[1.0, 0.0]]]])
    v = np.array([[[[2.0, 3.0]], [[5.0, 7.0]], [[-1.0, 4.0]]]])
    one, zero = np.ones((1, 3, 1)), np.zeros((1, 3, 1))
    o, S, _ = orc.delta_scan(k, k, v, zero, one, 1.0)
    assert np.allclose(o, v)
    assert np.allclose(S[0, 0], [[-1, 4], [5, 7]])


def test_delta_gradients_by_differences():
    s, reset, filled = _delta(0)
    r = np.random.default_rng(1)
    go, gs = r.normal(size=s["v"].shape), r.normal(size=s["s_first"].shape)
    names = ["q", "k", "v", "log_decay", "beta", "s_first"]

    def loss(d):
        o, S, _ = orc.delta_scan(d["q"], d["k"], d["v"], d["log_decay"], d["beta"], 0.7, reset, filled, d["s_first"])
        return (o * go).sum() + (S * gs).sum()

    grads = orc.delta_scan_grad(s["q"], s["k"], s["v"], s["log_decay"], s["beta"], 0.7, reset, filled, s["s_first"], go, gs)
    for name, g in zip(names, grads):
        for at in np.ndindex(g.shape):
            up, down = ({**s, name: s[name].copy()} for _ in range(2))
            up[name][at] += 1e-6
            down[name][at] -= 1e-6
            assert abs((loss(up) - loss(down)) / 2e-6 - g[at]) < 1e-7 * (1 + abs(g[at])) + 1e-8, (name, at)


def test_delta_step_is_one_step_of_the_scan():
    s, _, _ = _delta(3, T=1)
    o, S, _ = orc.delta_scan(s["q"], s["k"], s["v"], s["log_decay"], s["beta"], 0.5, None, None, s["s_first"])
    one = lambda n: s[n][:, 0]
    o1, table = orc.delta_step(one("q"), one("k"), one("v"), one("log_decay"), one("beta"), 0.5, None, None, s["s_first"])
    assert np.allclose(o1, o[:, 0]) and np.allclose(table, S)


@pytest.mark.parametrize("tail", [0, 1])
def test_distill_gradient_by_differences(tail):
    r = np.random.default_rng(2)
    R, V = 4, 7
    logits, avail = r.normal(size=(R, V)), np.ones((R, V), np.uint8)
    avail[1, 2] = avail[2, :4] = 0
    top_id = np.array([[1, 3, -1], [2, 0, 5], [5, 5, 6], [6, 7, 0]], np.int32)
    value = np.log(np.array([[0.5, 0.3, 0.1], [0.4, 0.3, 0.2], [0.4, 0.2, 0.3], [0.6, 0.1, 0.1]]))
    up = r.normal(size=R)
    grad = orc.distill(logits, top_id, value, avail, 1.3, tail, up)["grad"]
    for at in np.ndindex(R, V):
        d = np.zeros((R, V))
        d[at] = 1e-6
        diff = ((orc.distill(logits + d, top_id, value, avail, 1.3, tail)["loss"] - orc.distill(logits - d, top_id, value, avail, 1.3, tail)["loss"]) * up).sum() / 2e-6
        assert abs(diff - grad[at]) < 1e-8, at


def test_distill_of_oneself_is_zero():
    logits = np.random.default_rng(4).normal(size=(3, 9)) * 2
    top = policy_oracle.log_prob(logits, None, None, 0.8, K=4)
    both = orc.distill(logits, top["top_id"], top["top_logp"], None, 0.8, 1, np.ones(3))
    assert np.abs(both["loss"]).max() < 1e-12 and np.abs(both["grad"]).max() < 1e-12


def test_penalties_by_hand():
    logits = np.array([[2.0, -2.0, 1.0, 0.5]])
    out = orc.penalize(logits, np.array([[0, 1, 1, 9, 2]]), np.array([4]), np.array([1]), np.array([2.0]), np.array([0.25]), np.array([0.125]),
                       np.array([[3, 3, -1]]), np.array([[1.0, 0.5, 8.0]]), np.array([0b1011]))
    assert np.array_equal(out, [[1.0, -4.0 - 0.25 - 0.25, -np.inf, 2.0]])


# ------------------------------------------------------------------------------------------------ refusals



@pytest.fixture(scope="module")
def lib():
    import os
    if not os.path.exists(binding.LIB_PATH):
        from paper_2205_05248_amd import build
        build.build(verbose=False)
    return binding.load()


def _codes():
    import re
    import os
    text = open(os.path.join(os.path.dirname(__file__), "..", "include", "marl_qnet.h")).read()
    return {m.group(1): int(m.group(2)) for m in re.finditer(r"(MARL_ERR_\w+)\s*=?\s*\(?(-\d+)", text)}


P = 1 << 20                                     # an address that is never followed: every call here is refused


def _scan(lib, **k):
    d = dict(dtype=0, B=2, T=3, Hk=1, Hv=2, Dk=4, Dv=4, q=P, ld_q=4, k=2 * P, ld_k=4, v=3 * P, ld_v=8, g=4 * P, beta=5 * P, scale=1.0, reset=0,
             filled=0, s_first=0, o=6 * P, ld_o=8, s_last=0, keep=0, ws=8 * P, bytes=1 << 30, stream=0)
    d.update(k)
    return lib.marl_delta_scan(*d.values())


def _scan_grad(lib, **k):
    d = dict(dtype=0, B=2, T=3, Hk=1, Hv=2, Dk=4, Dv=4, q=P, ld_q=4, k=2 * P, ld_k=4, v=3 * P, ld_v=8, g=4 * P, beta=5 * P, scale=1.0, reset=0,
             filled=0, go=6 * P, ld_go=8, gs=0, ws=8 * P, bytes=1 << 30, gq=9 * P, ld_gq=4, gk=10 * P, ld_gk=4, gv=11 * P, ld_gv=8, gg=12 * P,
             gb=13 * P, gf=0, stream=0)
    d.update(k)
    return lib.marl_delta_scan_grad(*d.values())


def _step(lib, **k):
    d = dict(dtype=0, n=2, Hk=1, Hv=2, Dk=4, Dv=4, q=P, ld_q=4, k=2 * P, ld_k=4, v=3 * P, ld_v=8, g=4 * P, beta=5 * P, scale=1.0, slot=0, slots=2,
             reset=0, s_in=6 * P, s_out=6 * P, o=7 * P, ld_o=8, stream=0)
    d.update(k)
    return lib.marl_delta_step(*d.values())


def _distill(lib, **k):
    d = dict(dtype=0, R=2, V=5, K=2, logits=P, ld=5, ids=2 * P, values=3 * P, avail=0, ld_avail=0, scale=1.0, tail=1, loss=4 * P, log_sum=0, log_rest=0,
             ws=0, bytes=0, stream=0)
    d.update(k)
    return lib.marl_distill(*d.values())


def _distill_grad(lib, **k):
    d = dict(dtype=0, R=2, V=5, K=2, logits=P, ld=5, ids=2 * P, values=3 * P, avail=0, ld_avail=0, scale=1.0, tail=1, log_sum=4 * P, log_rest=5 * P,
             grad_loss=6 * P, out=7 * P, ld_out=5, stream=0)
    d.update(k)
    return lib.marl_distill_grad(*d.values())


def _penalize(lib, **k):
    d = dict(dtype=0, R=2, V=40, logits=P, ld=40, L=3, history=2 * P, ld_history=3, length=0, prompt=0, rep=0, pres=0, freq=0, M=1, ids=3 * P,
             values=4 * P, allowed=5 * P, ld_allowed=2, out=6 * P, ld_out=40, stream=0)
    d.update(k)
    return lib.marl_penalize(*d.values())


INF = float("inf")
REFUSED = [
    (_scan, "BAD_DTYPE", dict(dtype=3)), (_scan, "BAD_DIM", dict(Dk=129)), (_scan, "BAD_DIM", dict(Dk=0)), (_scan, "BAD_DIM", dict(Dv=1025)),
    (_scan, "BAD_DIM", dict(Hk=2, Hv=3)), (_scan, "BAD_DIM", dict(Hk=0)), (_scan, "BAD_DIM", dict(B=-1)), (_scan, "BAD_DIM", dict(T=-1)),
    (_scan, "BAD_DIM", dict(B=1 << 23)), (_scan, "BAD_DIM", dict(ld_q=3)), (_scan, "BAD_DIM", dict(ld_k=3)), (_scan, "BAD_DIM", dict(ld_v=7)),
    (_scan, "BAD_DIM", dict(ld_o=7)), (_scan, "BAD_DIM", dict(ld_o=1 << 31)), (_scan, "BAD_DIM", dict(bytes=100)), (_scan, "BAD_ARG", dict(scale=INF)),
    (_scan, "BAD_ARG", dict(ws=8 * P + 128)), (_scan, "BAD_ARG", dict(o=3 * P)),
    *[(_scan, "NULL", {n: 0}) for n in ("q", "k", "v", "g", "beta", "o", "ws")],
    *[(_scan_grad, "NULL", {n: 0}) for n in ("q", "k", "v", "g", "beta", "go", "gq", "gk", "gv", "gg", "gb", "ws")],
    *[(_scan_grad, "BAD_DIM", {n: 3}) for n in ("ld_q", "ld_k", "ld_v", "ld_go", "ld_gq", "ld_gk", "ld_gv", "bytes")],
    (_scan_grad, "BAD_ARG", dict(gq=P)), (_scan_grad, "BAD_ARG", dict(gk=9 * P)), (_scan_grad, "BAD_ARG", dict(gv=6 * P)),
    (_scan_grad, "BAD_ARG", dict(scale=float("nan"))), (_scan_grad, "BAD_ARG", dict(ws=8 * P + 4)), (_scan_grad, "BAD_DTYPE", dict(dtype=-1)),
    (_step, "BAD_DTYPE", dict(dtype=7)), (_step, "BAD_DIM", dict(n=3)), (_step, "BAD_DIM", dict(slots=0)), (_step, "BAD_DIM", dict(n=-1)),
    (_step, "BAD_DIM", dict(ld_o=7)), (_step, "BAD_DIM", dict(Dk=200)), (_step, "BAD_ARG", dict(o=P)), (_step, "BAD_ARG", dict(scale=INF)),
    *[(_step, "NULL", {n: 0}) for n in ("q", "k", "v", "g", "beta", "s_in", "s_out", "o")],
    (_distill, "BAD_DTYPE", dict(dtype=5)), (_distill, "BAD_DIM", dict(K=0)), (_distill, "BAD_DIM", dict(K=65)), (_distill, "BAD_DIM", dict(ld=4)),
    (_distill, "BAD_DIM", dict(V=0)), (_distill, "BAD_ARG", dict(scale=0.0)), (_distill, "BAD_DIM", dict(avail=9 * P, ld_avail=4)),
    (_distill, "BAD_DIM", dict(V=100000, ld=100000)), (_distill, "BAD_ARG", dict(V=100000, ld=100000, ws=P + 8, bytes=1 << 20)),
    *[(_distill, "NULL", {n: 0}) for n in ("logits", "ids", "values", "loss")],
    *[(_distill_grad, "NULL", {n: 0}) for n in ("logits", "ids", "values", "log_sum", "log_rest", "grad_loss", "out")],
    (_distill_grad, "BAD_DIM", dict(ld_out=4)), (_distill_grad, "BAD_ARG", dict(out=P, ld_out=6)), (_distill_grad, "BAD_DIM", dict(K=65)),
    (_penalize, "BAD_DTYPE", dict(dtype=4)), (_penalize, "BAD_DIM", dict(V=0)), (_penalize, "BAD_DIM", dict(ld=39)), (_penalize, "BAD_DIM", dict(ld_out=39)),
    (_penalize, "BAD_DIM", dict(ld_history=2)), (_penalize, "BAD_DIM", dict(ld_allowed=1)), (_penalize, "BAD_DIM", dict(M=1025)),
    (_penalize, "BAD_DIM", dict(L=1 << 24)), (_penalize, "BAD_DIM", dict(R=1 << 24)), (_penalize, "BAD_ARG", dict(out=P, ld_out=48)),
    (_scan, "BAD_DIM", dict(B=1 << 12, Hv=1024, ld_v=4096, ld_o=4096, T=128)), (_scan, "BAD_DIM", dict(B=1 << 12, T=1, Hv=1024, Dv=64, ld_v=1 << 16, ld_o=1 << 16)),
    (_scan_grad, "BAD_DIM", dict(B=1 << 12, T=1, Hv=1024, Dv=64, ld_v=1 << 16, ld_go=1 << 16, ld_gv=1 << 16)),
    (_step, "BAD_DIM", dict(n=1 << 13, slots=1 << 13, Hv=1024, Dv=64, ld_v=1 << 16, ld_o=1 << 16)),
    (_distill, "BAD_DIM", dict(R=1 << 26)), (_distill, "BAD_DIM", dict(R=1 << 24, V=2049, ld=2049)), (_distill_grad, "BAD_DIM", dict(R=1 << 26)),
    (_distill_grad, "BAD_DIM", dict(R=1 << 24, V=2049, ld=2049, ld_out=2049)), (_penalize, "BAD_DIM", dict(R=1 << 23, V=961, ld=961, ld_out=961, ld_allowed=31)),
    *[(_penalize, "NULL", {n: 0}) for n in ("logits", "history", "ids", "values", "out")],
]


@pytest.mark.parametrize("call,code,change", REFUSED)
def test_refusals(lib, call, code, change):
    assert call(lib, **change) == _codes()["MARL_ERR_" + code], change


def test_nothing_to_do_is_accepted(lib):
    assert _scan(lib, B=0) == 0 and _scan_grad(lib, B=0) == 0 and _step(lib, n=0) == 0
    assert _distill(lib, R=0) == 0 and _distill_grad(lib, R=0) == 0 and _penalize(lib, R=0) == 0


def test_workspace_sizes(lib):
    small, kept = (binding.marl_delta_scan_workspace_bytes("bf16", 2, 100, 1, 2, 64, 64, keep) for keep in (False, True))
    assert 0 < small < kept and small % 256 == 0 and kept % 256 == 0
    assert binding.marl_delta_scan_workspace_bytes("fp32", 0, 100, 1, 2, 64, 64) == 0 == binding.marl_delta_scan_workspace_bytes("fp32", 3, 0, 1, 2, 64, 64, True)
    assert binding.marl_distill_workspace_bytes(100, 2048, 5) == 0 < binding.marl_distill_workspace_bytes(1, 100000, 5)
    for bad in (dict(B=-1), dict(Dk=129), dict(Hv=3, Hk=2)):
        a = {**dict(B=2, T=3, Hk=1, Hv=2, Dk=4, Dv=4), **bad}
        with pytest.raises(binding.MarlError):
            binding.marl_delta_scan_workspace_bytes("fp32", a["B"], a["T"], a["Hk"], a["Hv"], a["Dk"], a["Dv"])
    n = ctypes.c_size_t()
    assert lib.marl_distill_workspace_bytes(1, 5, 0, ctypes.byref(n)) < 0 and lib.marl_distill_workspace_bytes(1, 5, 1, None) < 0
