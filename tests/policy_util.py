"""Helpers of the policy operators' GPU tests: seeded tensors, comparison with the 64-bit oracle."""
import numpy as np
import torch

DT = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def gen(seed):
    return torch.Generator().manual_seed(seed)


def randn(g, *shape, dtype=torch.float32):
    return torch.randn(*shape, generator=g).to(dtype)


def host(t):
    return None if t is None else t.double().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def half_step(dtype):
    """Rounding to nearest is off by at most this much of the value; nothing is rounded for fp32 outputs of fp32 sums."""
    return torch.finfo(dtype).eps / 2


def near(got, want, dtype, rel, name, floor=None):
    """|got - want| <= half a step of the type + `rel` of the largest wanted value (or of `floor`, an array or number)."""
    g = host(got)
    assert g.shape == want.shape, (name, g.shape, want.shape)
    assert (np.isfinite(g) == np.isfinite(want)).all(), f"{name}: finite in different places"
    ok = np.isfinite(want)
    assert (g[~ok] == want[~ok]).all(), f"{name}: infinities differ"
    if not ok.any():
        return
    scale = np.abs(want[ok]).max() if floor is None else floor
    tol = np.zeros(want.shape) + rel * scale + half_step(dtype) * np.abs(want) * (1 + 1e-6) + (
        torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps)
    err = np.zeros(want.shape)
    err[ok] = np.abs(g[ok] - want[ok])
    bad = ok & ~(err <= tol)
    if bad.any():
        k = np.unravel_index(np.argmax(np.where(ok, err / tol, 0)), want.shape)
        raise AssertionError(f"{name}: {bad.sum()} of {bad.size} off, worst at {k}: {g[k]} for {want[k]}, allowed {tol[k]}")
