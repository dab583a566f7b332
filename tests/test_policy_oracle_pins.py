"""The oracle of the policy operators against closed forms and differences, and the library's refusals (CPU only)."""
import ctypes

import numpy as np
import pytest

from oracle import policy_oracle as orc
from paper_2205_05248_amd import binding


@pytest.fixture(scope="module")
def lib():
    import os
    if not os.path.exists(binding.LIB_PATH):
        from paper_2205_05248_amd import build
        build.build(verbose=False)
    return binding.load()


def _difference(f, v, k, step=1e-6):
    up, down = v.copy(), v.copy()
    up.flat[k] += step
    down.flat[k] -= step
    return (f(up) - f(down)) / (2 * step)


def test_recurrence_with_constant_gates_is_a_geometric_sum():
    T, C = 7, 3
    lam = np.array([-2.0, 0.0, 1.0])
    rate = 8 * np.log1p(np.exp(lam))
    a = np.exp(-rate * 0.5)
    y, last, _ = orc.linear_scan(np.ones((1, T, C)), np.zeros((1, T, C)), np.zeros((1, T, C)), lam, 8.0, h_first=np.full((1, C), 2.0))
    want = np.stack([2 * a ** (t + 1) + 0.5 * np.sqrt(1 - a * a) * (1 - a ** (t + 1)) / (1 - a) for t in range(T)])
    assert np.abs(y[0] - want).max() < 1e-14 and np.abs(last[0] - want[-1]).max() < 1e-14


def test_recurrence_padding_and_resets():
    g = np.random.default_rng(0)
    x, r, i = (g.normal(size=(2, 6, 4)) for _ in range(3))
    lam, h0 = g.normal(size=4), g.normal(size=(2, 4))
    filled = np.array([[1, 0, 1, 1, 0, 1], [0] * 6])
    reset = np.array([[0, 1, 0, 1, 0, 0], [1] * 6])
    y, last, _ = orc.linear_scan(x, r, i, lam, 8.0, reset, filled, h0)
    assert (y[filled == 0] == 0).all() and (last[1] == h0[1]).all()
    keep = [0, 2, 3, 5]                                            # padding taken out: the same sequence
    z, zlast, _ = orc.linear_scan(x[:1, keep], r[:1, keep], i[:1, keep], lam, 8.0, reset[:1, keep], None, h0[:1])
    assert np.array_equal(z[0], y[0, keep]) and np.array_equal(zlast[0], last[0])
    w, _, _ = orc.linear_scan(x[:1, 3:4], r[:1, 3:4], i[:1, 3:4], lam, 8.0, np.array([[1]]))     # nothing of before is left
    assert np.array_equal(w[0, 0], y[0, 3])


def test_recurrence_gradient_against_differences():
    g = np.random.default_rng(1)
    B, T, C = 2, 5, 3
    x, r, i, gy = (g.normal(size=(B, T, C)) for _ in range(4))
    lam, h0, gl = g.normal(size=C), g.normal(size=(B, C)), g.normal(size=(B, C))
    filled = np.array([[1, 1, 0, 1, 1], [1, 0, 0, 1, 1]])
    reset = np.array([[0, 0, 0, 1, 0], [0, 1, 0, 0, 0]])

    def loss(x=x, r=r, i=i, lam=lam, h0=h0):
        y, last, _ = orc.linear_scan(x, r, i, lam, 8.0, reset, filled, h0)
        return (y * gy).sum() + (last * gl).sum()

    got = orc.linear_scan_grad(x, r, i, lam, 8.0, reset, filled, h0, gy, gl)
    for grad, name, v in zip(got, ("x", "r", "i", "lam", "h0"), (x, r, i, lam, h0)):
        for k in range(v.size):
            want = _difference(lambda u: loss(**{name: u}), v, k)
            assert abs(grad.flat[k] - want) < 1e-7 * max(1.0, abs(want)), (name, k)


def test_log_prob_of_equal_logits_and_its_masks():
    logits = np.zeros((3, 5))
    logits[2, 1] = -np.inf
    avail = np.array([[1, 1, 0, 1, 1], [0] * 5, [0, 1, 1, 0, 0]])
    logits[0, 2] = np.nan                                          # masked: not looked at
    out = orc.log_prob(logits, np.array([1, 2, 1]), avail, 1.0, K=3)
    assert np.allclose(out["logp"][:2], [-np.log(4), 0.0]) and out["logp"][2] == -np.inf
    assert np.allclose(out["entropy"], [np.log(4), 0.0, 0.0])
    assert out["top_id"].tolist() == [[0, 1, 3], [-1, -1, -1], [2, -1, -1]]


def test_log_prob_gradient_against_differences():
    g = np.random.default_rng(2)
    logits, avail = g.normal(size=(4, 6)), (g.random((4, 6)) < 0.7).astype(np.uint8)
    token = np.array([0, 3, -1, 5])
    avail[0, 0] = avail[1, 3] = 1
    avail[3, 5] = 0                                                # not available: no gradient through logp
    gl, ge = g.normal(size=4), g.normal(size=4)

    def loss(l):
        out = orc.log_prob(l, token, avail, 0.7)
        return (np.where(np.isfinite(out["logp"]), out["logp"], 0) * gl).sum() + (out["entropy"] * ge).sum()

    grad = orc.log_prob_grad(logits, token, avail, 0.7, gl, ge)
    for k in range(logits.size):
        assert abs(grad.flat[k] - _difference(loss, logits, k)) < 1e-8


def test_newton_schulz_maps_singular_values_by_its_polynomial():
    g = np.random.default_rng(3)
    u, _ = np.linalg.qr(g.normal(size=(5, 5)))
    v, _ = np.linalg.qr(g.normal(size=(9, 9)))
    s = np.array([3.0, 2.0, 1.0, 0.5, 0.01])
    m = u @ np.diag(s) @ v[:5]
    t = s / np.linalg.norm(s)
    for _ in range(5):
        t = 3.4445 * t - 4.7750 * t ** 3 + 2.0315 * t ** 5
    assert np.abs(orc.orthogonalize(m) - u @ np.diag(t) @ v[:5]).max() < 1e-12
    assert np.abs(orc.orthogonalize(m.T) - orc.orthogonalize(m).T).max() < 1e-12
    assert (orc.orthogonalize(np.zeros((3, 4))) == 0).all()


# ---------------------------------------------------------------------------------------------- refusals of the C ABI
P = 0x100000                                                       # an address that no refused call reaches
F32 = binding.MARL_DTYPE_F32


def _scan(lib, **k):
    a = dict(dtype=F32, B=1, T=2, C=4, x=P, ld_x=4, r=P, ld_r=4, i=P, ld_i=4, lam=P, decay=8.0, reset=None, filled=None, h_first=None,
             y=P + 4096, ld_y=4, h_last=None, ws=P, ws_bytes=1 << 20, stream=None)
    a.update(k)
    return lib.marl_linear_scan(*a.values())


def _scan_grad(lib, **k):
    a = dict(dtype=F32, B=1, T=2, C=4, x=P, ld_x=4, r=P, ld_r=4, i=P, ld_i=4, lam=P, decay=8.0, reset=None, filled=None, gy=P, ld_gy=4,
             gl=None, ws=P, ws_bytes=1 << 20, gx=P + 256, ld_gx=4, gr=P + 512, ld_gr=4, gi=P + 768, ld_gi=4, glam=P, gh=None, stream=None)
    a.update(k)
    return lib.marl_linear_scan_grad(*a.values())


def _step(lib, **k):
    a = dict(dtype=F32, n=2, C=4, x=P, ld_x=4, r=P, ld_r=4, i=P, ld_i=4, lam=P, decay=8.0, slot=None, slots=2, reset=None, h_in=P, h_out=P,
             y=P + 256, ld_y=4, stream=None)
    a.update(k)
    return lib.marl_linear_step(*a.values())


def _logp(lib, **k):
    a = dict(dtype=F32, R=2, V=4, logits=P, ld=4, token=P, avail=None, ld_avail=0, scale=1.0, logp=P, entropy=P, log_sum=P, K=0, top_id=None,
             top_logp=None, ws=P, ws_bytes=1 << 20, stream=None)
    a.update(k)
    return lib.marl_log_prob(*a.values())


def _logp_grad(lib, **k):
    a = dict(dtype=F32, R=2, V=4, logits=P, ld=4, token=P, avail=None, ld_avail=0, scale=1.0, log_sum=P, entropy=P, gl=P, ge=P, out=P + 256,
             ld_grad=4, stream=None)
    a.update(k)
    return lib.marl_log_prob_grad(*a.values())


COEF = (ctypes.c_float * 3)(3.4445, -4.775, 2.0315)


def _ortho(lib, **k):
    a = dict(dtype=F32, L=1, rows=4, cols=4, m=P, out=P, ws=P, ws_bytes=1 << 30, steps=5, coef=COEF, eps=1e-7, stream=None)
    a.update(k)
    return lib.marl_orthogonalize(*a.values())


def _muon(lib, **k):
    a = dict(dtype=F32, L=1, rows=4, cols=4, w=P, g=P, m=P, wo=P, mo=P, ws=P, ws_bytes=1 << 30, lr=0.1, beta=0.9, nesterov=1, wd=0.0, scale=1.0,
             steps=5, coef=COEF, eps=1e-7, stream=None)
    a.update(k)
    return lib.marl_muon_step(*a.values())


NULL, DIM, TYPE, ARG = -1, -2, -3, -5
NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("call,change,want", [
    (_scan, dict(dtype=3), TYPE), (_scan, dict(dtype=-1), TYPE), (_scan, dict(B=-1), DIM), (_scan, dict(T=-1), DIM), (_scan, dict(C=-1), DIM),
    (_scan, dict(C=1 << 24), DIM), (_scan, dict(B=1 << 20, T=1 << 20), DIM), (_scan, dict(ld_x=3), DIM), (_scan, dict(ld_y=3), DIM),
    (_scan, dict(x=None), NULL), (_scan, dict(r=None), NULL), (_scan, dict(i=None), NULL), (_scan, dict(lam=None), NULL), (_scan, dict(y=None), NULL),
    (_scan, dict(ws=None), NULL), (_scan, dict(ws_bytes=8), DIM), (_scan, dict(ws=P + 16), ARG), (_scan, dict(y=P), ARG),
    (_scan, dict(decay=0.0), ARG), (_scan, dict(decay=NAN), ARG), (_scan, dict(decay=INF), ARG), (_scan, dict(B=0), 0), (_scan, dict(C=0), 0),
    (_scan_grad, dict(dtype=7), TYPE), (_scan_grad, dict(T=-2), DIM), (_scan_grad, dict(ld_gx=3), DIM), (_scan_grad, dict(ld_gy=1), DIM),
    (_scan_grad, dict(gy=None), NULL), (_scan_grad, dict(glam=None), NULL), (_scan_grad, dict(gr=None), NULL), (_scan_grad, dict(ws_bytes=0), DIM),
    (_scan_grad, dict(gx=P), ARG), (_scan_grad, dict(gi=P + 256), ARG), (_scan_grad, dict(ws=P + 64), ARG), (_scan_grad, dict(decay=-1.0), ARG),
    (_scan_grad, dict(C=0), 0),
    (_step, dict(dtype=9), TYPE), (_step, dict(n=-1), DIM), (_step, dict(slots=0), DIM), (_step, dict(slots=1), DIM), (_step, dict(ld_i=2), DIM),
    (_step, dict(h_in=None), NULL), (_step, dict(y=None), NULL), (_step, dict(y=P), ARG), (_step, dict(decay=0.0), ARG), (_step, dict(n=0), 0),
    (_logp, dict(dtype=3), TYPE), (_logp, dict(V=0), DIM), (_logp, dict(R=-1), DIM), (_logp, dict(V=1 << 30), DIM), (_logp, dict(ld=3), DIM),
    (_logp, dict(K=65), DIM), (_logp, dict(K=-1), DIM), (_logp, dict(avail=P, ld_avail=2), DIM), (_logp, dict(logits=None), NULL),
    (_logp, dict(token=None), NULL), (_logp, dict(K=2), NULL), (_logp, dict(scale=0.0), ARG), (_logp, dict(scale=-1.0), ARG),
    (_logp, dict(scale=INF), ARG), (_logp, dict(ws=P + 4), ARG), (_logp, dict(R=0), 0),
    (_logp_grad, dict(dtype=3), TYPE), (_logp_grad, dict(ld_grad=3), DIM), (_logp_grad, dict(out=P, ld=5), ARG), (_logp_grad, dict(out=None), NULL),
    (_logp_grad, dict(log_sum=None), NULL), (_logp_grad, dict(entropy=None), NULL), (_logp_grad, dict(token=None), NULL),
    (_logp_grad, dict(scale=NAN), ARG), (_logp_grad, dict(R=0), 0),
    (_ortho, dict(dtype=3), TYPE), (_ortho, dict(L=-1), DIM), (_ortho, dict(rows=0), DIM), (_ortho, dict(cols=32769), DIM), (_ortho, dict(m=None), NULL),
    (_ortho, dict(out=None), NULL), (_ortho, dict(coef=None), NULL), (_ortho, dict(ws=None), NULL), (_ortho, dict(ws_bytes=16), DIM),
    (_ortho, dict(steps=-1), ARG), (_ortho, dict(steps=65), ARG), (_ortho, dict(eps=0.0), ARG), (_ortho, dict(coef=(ctypes.c_float * 3)(1, NAN, 1)), ARG),
    (_ortho, dict(ws=P + 8), ARG), (_ortho, dict(L=0), 0),
    (_muon, dict(dtype=3), TYPE), (_muon, dict(g=None), NULL), (_muon, dict(m=None), NULL), (_muon, dict(wo=None), NULL), (_muon, dict(lr=NAN), ARG),
    (_muon, dict(beta=INF), ARG), (_muon, dict(wd=NAN), ARG), (_muon, dict(scale=INF), ARG), (_muon, dict(ws_bytes=1), DIM), (_muon, dict(L=0), 0),
])
def test_refusals_come_before_the_device_is_used(lib, call, change, want):
    assert call(lib, **change) == want


def test_workspace_sizes(lib):
    n = ctypes.c_size_t()
    assert lib.marl_linear_scan_workspace_bytes(F32, 2, 3, 4, None) == NULL
    assert lib.marl_linear_scan_workspace_bytes(5, 2, 3, 4, ctypes.byref(n)) == TYPE
    assert lib.marl_linear_scan_workspace_bytes(F32, -2, 3, 4, ctypes.byref(n)) == DIM
    assert lib.marl_log_prob_workspace_bytes(4, 0, 0, ctypes.byref(n)) == DIM
    assert lib.marl_log_prob_workspace_bytes(4, 10, 65, ctypes.byref(n)) == DIM
    assert lib.marl_muon_workspace_bytes(F32, 1, 0, 4, ctypes.byref(n)) == DIM
    assert lib.marl_muon_workspace_bytes(F32, 1, 4, 4, None) == NULL
    with pytest.raises(ValueError):
        binding.marl_muon_workspace_bytes("fp8", 1, 4, 4)
    assert binding.marl_linear_scan_workspace_bytes("bf16", 0, 0, 0) >= 0


def test_binding_refuses_tensors_of_the_wrong_kind():
    import torch
    x = torch.zeros(1, 2, 4)                                       # on the host
    with pytest.raises(ValueError):
        binding.marl_linear_scan(x, x, x, torch.zeros(4), 8.0, None, None, None, x, None, None)
    with pytest.raises(ValueError):
        binding.marl_log_prob(x[0].double(), None, None, 1.0, None, None, None)
    with pytest.raises(ValueError):
        binding.marl_orthogonalize(torch.zeros(4), torch.zeros(4), None)
    with pytest.raises(ValueError):
        binding.marl_orthogonalize(torch.zeros(4, 4), torch.zeros(4, 4), None)


@pytest.mark.parametrize("call", [_scan, _scan_grad])
@pytest.mark.parametrize("name", ["ld_x", "ld_r", "ld_i"])
def test_rows_of_the_scans_that_lie_too_far_apart_are_refused(lib, call, name):
    """A lane's offset inside a wave's rows has 32 bits."""
    assert call(lib, **{name: 1 << 27}) == DIM
    assert call(lib, B=0, C=0, **{name: 1 << 27}) == 0


@pytest.mark.parametrize("call,names", [(_scan, ["ld_x", "ld_r", "ld_i", "ld_y"]), (_scan_grad, ["ld_x", "ld_r", "ld_i", "ld_gy", "ld_gx", "ld_gr", "ld_gi"])])
@pytest.mark.parametrize("below", [1, 2, 3, 63])
def test_the_widest_rows_leave_room_for_a_lanes_channel(lib, call, names, below):
    """16 rows of 16-bit elements and the channel of a lane, up to 62, are one 32-bit offset: just below 2^27 elements it would wrap."""
    worst = 16 * (2 ** 27 - 64) * 2 + 62 * 2 + 4
    assert worst <= 2 ** 32 < 16 * (2 ** 27 - 1) * 2 + 62 * 2 + 4
    for name in names:
        assert call(lib, dtype=binding.MARL_DTYPE_BF16, **{name: 2 ** 27 - below}) == DIM, name
