"""The policy operators in 64 bits with numpy: gated linear recurrence, log probabilities, Newton-Schulz update.

Written from the formulas in include/marl_qnet.h, one step or one row at a time, with no code in common with the
library."""
import numpy as np


def _sigmoid(v):
    v = np.asarray(v, np.float64)
    e = np.exp(-np.abs(v))
    return np.where(v >= 0, 1 / (1 + e), e / (1 + e))


def rates(lam, decay):
    """Decay rate per unit of gate, and its derivative by lam."""
    lam = np.asarray(lam, np.float64)
    return decay * np.logaddexp(0.0, lam), decay * _sigmoid(lam)


def _gates(r, i, rate):
    s_r, s_i = _sigmoid(r), _sigmoid(i)
    L = -rate * s_r
    return s_r, s_i, np.exp(L), np.sqrt(-np.expm1(2 * L))


def linear_scan(x, r, i, lam, decay, reset=None, filled=None, h_first=None):
    """y, h_last and the states before every step."""
    x, r, i = (np.asarray(v, np.float64) for v in (x, r, i))
    B, T, C = x.shape
    rate, _ = rates(lam, decay)
    y, before = np.zeros((B, T, C)), np.zeros((B, T, C))
    h_last = np.zeros((B, C)) if h_first is None else np.array(h_first, np.float64)
    for b in range(B):
        h = h_last[b].copy()
        for t in range(T):
            before[b, t] = h
            if filled is not None and not filled[b, t]:
                continue
            s_r, s_i, a, beta = _gates(r[b, t], i[b, t], rate)
            h = s_i * x[b, t] if reset is not None and reset[b, t] else a * h + beta * s_i * x[b, t]
            y[b, t] = h
        h_last[b] = h
    return y, h_last, before


def linear_scan_grad(x, r, i, lam, decay, reset, filled, h_first, grad_y, grad_h_last=None):
    """grad_x, grad_r, grad_i, grad_lam, grad_h_first."""
    _, _, before = linear_scan(x, r, i, lam, decay, reset, filled, h_first)
    x, r, i, grad_y = (np.asarray(v, np.float64) for v in (x, r, i, grad_y))
    B, T, C = x.shape
    rate, rate_by_lam = rates(lam, decay)
    gx, gr, gi = (np.zeros((B, T, C)) for _ in range(3))
    by_rate = np.zeros(C)
    dh_first = np.zeros((B, C)) if grad_h_last is None else np.array(grad_h_last, np.float64)
    for b in range(B):
        dh = dh_first[b].copy()
        for t in range(T - 1, -1, -1):
            if filled is not None and not filled[b, t]:
                continue
            dh = dh + grad_y[b, t]
            s_r, s_i, a, beta = _gates(r[b, t], i[b, t], rate)
            if reset is not None and reset[b, t]:
                gx[b, t] = dh * s_i
                gi[b, t] = dh * x[b, t] * s_i * (1 - s_i)
                dh = np.zeros(C)
                continue
            gx[b, t] = dh * beta * s_i
            gi[b, t] = dh * beta * x[b, t] * s_i * (1 - s_i)
            by_a = dh * before[b, t]
            by_beta = dh * s_i * x[b, t]
            by_L = by_a * a - by_beta * a * a / beta
            gr[b, t] = by_L * -rate * s_r * (1 - s_r)
            by_rate -= by_L * s_r
            dh = a * dh
        dh_first[b] = dh
    return gx, gr, gi, by_rate * rate_by_lam, dh_first


def linear_step(x, r, i, lam, decay, slot, reset, h_in):
    """y and the table afterwards."""
    h_out = np.array(h_in, np.float64)
    n = len(x)
    y = np.zeros((n, h_out.shape[1]))
    for k in range(n):
        s = k if slot is None else int(slot[k])
        one = None if reset is None else np.array([[reset[k]]])
        out, last, _ = linear_scan(x[k][None, None], r[k][None, None], i[k][None, None], lam, decay, one, None, np.asarray(h_in)[s][None])
        y[k], h_out[s] = out[0, 0], last[0]
    return y, h_out


def log_prob(logits, token, avail, scale, K=0):
    """dict of logp, entropy, log_sum, top_id, top_logp; avail [V], [R,V] or None."""
    R, V = logits.shape
    out = dict(logp=np.zeros(R), entropy=np.zeros(R), log_sum=np.full(R, -np.inf), top_id=np.full((R, K), -1, np.int32),
               top_logp=np.full((R, K), -np.inf))
    for k in range(R):
        raw = np.asarray(logits[k], np.float64)
        ok = np.ones(V, bool) if avail is None else (avail if avail.ndim == 1 else avail[k]) != 0
        ok = ok & ~(raw == -np.inf)
        index = np.flatnonzero(ok)
        if not len(index):
            continue
        z = scale * raw[index]
        top = z.max()
        log_sum = top + np.log(np.exp(z - top).sum())
        out["log_sum"][k] = log_sum
        p = np.exp(z - log_sum)
        out["entropy"][k] = -(p * (z - log_sum)).sum()
        if token is not None and 0 <= token[k] < V:
            out["logp"][k] = scale * raw[token[k]] - log_sum if ok[token[k]] else -np.inf
        order = index[np.lexsort((index, -raw[index]))][:K]
        out["top_id"][k, :len(order)] = order
        out["top_logp"][k, :len(order)] = scale * raw[order] - log_sum
    return out


def log_prob_grad(logits, token, avail, scale, grad_logp=None, grad_entropy=None):
    R, V = logits.shape
    fwd = log_prob(logits, token, avail, scale)
    grad = np.zeros((R, V))
    for k in range(R):
        if fwd["log_sum"][k] == -np.inf:
            continue
        raw = np.asarray(logits[k], np.float64)
        ok = np.ones(V, bool) if avail is None else (avail if avail.ndim == 1 else avail[k]) != 0
        index = np.flatnonzero(ok & ~(raw == -np.inf))
        lp = scale * raw[index] - fwd["log_sum"][k]
        p = np.exp(lp)
        g = np.zeros(len(index))
        if grad_logp is not None and token is not None and token[k] in index:
            g = grad_logp[k] * ((index == token[k]) - p)
        if grad_entropy is not None:
            g = g - grad_entropy[k] * p * (lp + fwd["entropy"][k])
        grad[k, index] = scale * g
    return grad


def orthogonalize(matrix, steps=5, coefficients=(3.4445, -4.7750, 2.0315), eps=1e-7):
    X = np.asarray(matrix, np.float64)
    if X.ndim == 3:
        return np.stack([orthogonalize(m, steps, coefficients, eps) for m in X])
    if X.shape[0] > X.shape[1]:
        return orthogonalize(X.T, steps, coefficients, eps).T
    X = X / max(np.linalg.norm(X), eps)
    for _ in range(steps):
        G = X @ X.T
        X = coefficients[0] * X + (coefficients[1] * G + coefficients[2] * (G @ G)) @ X
    return X


def muon_step(weights, grad, momentum, lr, beta, nesterov, weight_decay, scale, **ns):
    """weights and momentum afterwards."""
    grad = np.asarray(grad, np.float64)
    momentum = beta * np.asarray(momentum, np.float64) + grad
    u = grad + beta * momentum if nesterov else momentum
    return (1 - lr * weight_decay) * np.asarray(weights, np.float64) - lr * scale * orthogonalize(u, **ns), momentum
