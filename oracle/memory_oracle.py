"""Gated delta rule, distillation and logit penalties in 64 bits with numpy.

Written from the formulas in include/marl_qnet.h, one step, row or place at a time, with no code in common with the
library."""
import numpy as np


def _heads(t, Hv):
    """One row per value head: value head h reads key head h // (Hv // Hk)."""
    t = np.asarray(t, np.float64)
    return np.repeat(t, Hv // t.shape[-2], axis=-2)


def _decay(log_decay, reset):
    with np.errstate(under="ignore"):
        a = np.exp(np.maximum(np.asarray(log_decay, np.float64), -200.0))
    a = np.where(np.asarray(log_decay) == -np.inf, 0.0, a)
    return a if reset is None else np.where(np.asarray(reset)[..., None] != 0, 0.0, a)


def _dropped(a, S):
    """a S, nothing where a is 0."""
    return np.where(a == 0, 0.0, a * np.where(a == 0, 0.0, S))


def delta_scan(q, k, v, log_decay, beta, scale, reset=None, filled=None, s_first=None):
    """o, s_last and the states before every step."""
    v = np.asarray(v, np.float64)
    B, T, Hv, Dv = v.shape
    q, k, a = _heads(q, Hv), _heads(k, Hv), _decay(log_decay, reset)
    Dk = q.shape[-1]
    beta = np.asarray(beta, np.float64)
    S = np.zeros((B, Hv, Dk, Dv)) if s_first is None else np.array(s_first, np.float64)
    o, before = np.zeros((B, T, Hv, Dv)), np.zeros((B, T, Hv, Dk, Dv))
    for t in range(T):
        before[:, t] = S
        for b in range(B):
            if filled is not None and not filled[b, t]:
                continue
            for h in range(Hv):
                old = _dropped(a[b, t, h], S[b, h])
                u = beta[b, t, h] * (v[b, t, h] - old.T @ k[b, t, h])
                S[b, h] = old + np.outer(k[b, t, h], u)
                o[b, t, h] = scale * (S[b, h].T @ q[b, t, h])
    return o, S, before


def delta_scan_grad(q, k, v, log_decay, beta, scale, reset, filled, s_first, grad_o, grad_s_last=None):
    """grad_q, grad_k, grad_v, grad_log_decay, grad_beta, grad_s_first."""
    _, _, before = delta_scan(q, k, v, log_decay, beta, scale, reset, filled, s_first)
    Hk = np.asarray(q).shape[-2]
    v, grad_o = np.asarray(v, np.float64), np.asarray(grad_o, np.float64)
    B, T, Hv, Dv = v.shape
    q, k, a = _heads(q, Hv), _heads(k, Hv), _decay(log_decay, reset)
    Dk = q.shape[-1]
    gq, gk, gv = np.zeros((B, T, Hk, Dk)), np.zeros((B, T, Hk, Dk)), np.zeros((B, T, Hv, Dv))
    gg, gb = np.zeros((B, T, Hv)), np.zeros((B, T, Hv))
    D = np.zeros((B, Hv, Dk, Dv)) if grad_s_last is None else np.array(grad_s_last, np.float64)
    for b in range(B):
        for h in range(Hv):
            to = h // (Hv // Hk)
            for t in range(T - 1, -1, -1):
                if filled is not None and not filled[b, t]:
                    continue
                at, kt, bt = a[b, t, h], k[b, t, h], float(beta[b, t, h])
                old = _dropped(at, before[b, t, h])
                miss = v[b, t, h] - old.T @ kt
                u = bt * miss
                S = old + np.outer(kt, u)
                go = scale * grad_o[b, t, h]
                gq[b, t, to] += S @ go
                adj = D[b, h] + np.outer(q[b, t, h], go)
                du = adj.T @ kt
                gb[b, t, h] = du @ miss
                gv[b, t, h] = bt * du
                gk[b, t, to] += adj @ u - old @ (bt * du)
                d_old = adj - np.outer(kt, bt * du)
                gg[b, t, h] = (d_old * old).sum() if at != 0 else 0.0
                D[b, h] = _dropped(at, d_old)
    return gq, gk, gv, gg, gb, D


def delta_step(q, k, v, log_decay, beta, scale, slot, reset, s_in):
    """o and the table afterwards."""
    table = np.array(s_in, np.float64)
    o = np.zeros(np.asarray(v).shape)
    for i in range(len(o)):
        s = i if slot is None else int(slot[i])
        one = None if reset is None else np.array([[reset[i]]])
        out, last, _ = delta_scan(q[i][None, None], k[i][None, None], v[i][None, None], log_decay[i][None, None], beta[i][None, None], scale, one,
                                  None, np.asarray(s_in)[s][None])
        o[i], table[s] = out[0, 0], last[0]
    return o, table


def distill(logits, top_id, top_value, avail, scale, tail, grad_loss=None):
    """dict of loss, log_sum, log_rest and, with grad_loss, grad and the sum of the sizes of its terms."""
    logits = np.asarray(logits, np.float64)
    R, V = logits.shape
    out = dict(loss=np.zeros(R), log_sum=np.full(R, -np.inf), log_rest=np.full(R, -np.inf), grad=np.zeros((R, V)),
               grad_size=np.zeros((R, V)))
    for r in range(R):
        ok = np.ones(V, bool) if avail is None else (avail if avail.ndim == 1 else avail[r]) != 0
        ok = ok & ~(logits[r] == -np.inf)
        if not ok.any():
            continue
        z = scale * np.where(ok, logits[r], 0.0)
        top = z[ok].max()
        e = np.where(ok, np.exp(z - top), 0.0)
        log_sum = top + np.log(e.sum())
        q = e / e.sum()
        kept = [(int(i), float(x)) for i, x in zip(top_id[r], top_value[r]) if 0 <= i < V and ok[i]]
        target, loss, mass = np.zeros(V), 0.0, 0.0
        values = np.array([x for _, x in kept])
        if not tail and len(values) and np.isfinite(values).any():
            values = values - (values.max() + np.log(np.exp(values - values.max()).sum()))
        elif not tail:
            values = np.full(len(values), -np.inf)
        for (i, _), x in zip(kept, values):
            p = np.exp(x)
            mass += p
            target[i] += p
            if p > 0:
                loss += p * (x - (z[i] - log_sum))
        others = ok.copy()
        others[[i for i, _ in kept]] = False
        left = 0.0
        if tail and others.any():
            zo = z[others]
            out["log_rest"][r] = zo.max() + np.log(np.exp(zo - zo.max()).sum()) - log_sum
            left = max(0.0, 1.0 - mass)
            if left > 0:
                loss += left * (np.log(left) - out["log_rest"][r])
        out["loss"][r], out["log_sum"][r] = loss, log_sum
        if grad_loss is not None:
            g, size = (mass + left) * q - target, (mass + left) * q + target
            if left > 0:
                part = left * np.exp(z[others] - log_sum - out["log_rest"][r])
                g[others] -= part
                size[others] += part
            out["grad"][r] = np.where(ok, scale * float(grad_loss[r]) * g, 0.0)
            out["grad_size"][r] = np.where(ok, scale * abs(float(grad_loss[r])) * size, 0.0)
    return out


def penalize(logits, history=None, length=None, prompt=None, repetition=None, presence=None, frequency=None, bias_id=None, bias_value=None,
             allowed=None):
    out = np.array(logits, np.float64)
    R, V = out.shape
    for r in range(R):
        L = 0 if history is None else history.shape[1]
        n = L if length is None else min(max(int(length[r]), 0), L)
        start = 0 if prompt is None else min(max(int(prompt[r]), 0), n)
        seen, count = set(), {}
        for t in range(n):
            j = int(history[r, t])
            if 0 <= j < V:
                seen.add(j)
                if t >= start:
                    count[j] = count.get(j, 0) + 1
        for j in seen:
            if repetition is not None:
                rho = float(repetition[r])
                out[r, j] = out[r, j] / rho if out[r, j] > 0 else out[r, j] * rho
        for j, c in count.items():
            out[r, j] -= (0.0 if presence is None else float(presence[r])) + (0.0 if frequency is None else float(frequency[r])) * c
        for m in range(0 if bias_id is None else bias_id.shape[1]):
            j = int(bias_id[r, m])
            if 0 <= j < V:
                out[r, j] += float(bias_value[r, m])
        if allowed is not None:
            words = allowed if allowed.ndim == 1 else allowed[r]
            for j in range(V):
                if not (int(words[j // 32]) & 0xffffffff) >> (j % 32) & 1:
                    out[r, j] = -np.inf
    return out
