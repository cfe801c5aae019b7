"""Double-precision reference of the student's operators (test infrastructure): the gated delta rule token by
token with the gradient by the reverse recursion, the distillation loss with its gradient, the selection of the
largest logits.  NumPy only, written from the definitions in include/pql_student.h."""
from __future__ import annotations

import numpy as np


def delta_forward(q, k, v, g, beta, scale, lengths=None, state=None, keep=False):
    """q, k [n,t,hk,dk], v [n,t,hv,dv], g, beta [n,t,hv] -> out [n,t,hv,dv], state [n,hv,dk,dv] (and what the
    gradient needs)."""
    q, k, v, g, beta = (np.asarray(x, np.float64) for x in (q, k, v, g, beta))
    n, t, hk, dk = q.shape
    hv, dv = v.shape[2:]
    group = hv // hk
    out = np.zeros((n, t, hv, dv))
    S = np.zeros((n, hv, dk, dv)) if state is None else np.array(state, np.float64)
    kept = {}
    for b in range(n):
        length = t if lengths is None else min(max(int(lengths[b]), 0), t)
        for i in range(length):
            for h in range(hv):
                kk, qq = k[b, i, h // group], q[b, i, h // group]
                a = np.exp(g[b, i, h])
                before = a * S[b, h] if a != 0 else np.zeros((dk, dv))
                r = v[b, i, h] - kk @ before
                after = before + np.outer(kk, beta[b, i, h] * r)
                if keep:
                    kept[b, i, h] = (S[b, h].copy(), before, r, after)
                S[b, h] = after
                out[b, i, h] = scale * (qq @ after)
    return (out, S, kept) if keep else (out, S)


def delta_backward(q, k, v, g, beta, scale, out_grad, state_grad=None, lengths=None, state=None):
    """Gradients of sum(out * out_grad) + sum(state_out * state_grad): dq, dk, dv, dg, dbeta, dstate."""
    q, k, v, g, beta, do = (np.asarray(x, np.float64) for x in (q, k, v, g, beta, out_grad))
    _, S, kept = delta_forward(q, k, v, g, beta, scale, lengths, state, keep=True)
    n, t, hk, _ = q.shape
    hv = v.shape[2]
    group = hv // hk
    dq, dk, dv, dg, db = (np.zeros_like(x) for x in (q, k, v, g, beta))
    dS = np.zeros_like(S) if state_grad is None else np.array(state_grad, np.float64)
    for b in range(n):
        length = t if lengths is None else min(max(int(lengths[b]), 0), t)
        for i in reversed(range(length)):
            for h in range(hv):
                kk, qq = k[b, i, h // group], q[b, i, h // group]
                start, before, r, after = kept[b, i, h]
                d = dS[b, h] + scale * np.outer(qq, do[b, i, h])
                dq[b, i, h // group] += scale * (after @ do[b, i, h])
                du = kk @ d
                db[b, i, h] = du @ r
                dr = beta[b, i, h] * du
                dv[b, i, h] = dr
                dk[b, i, h // group] += d @ (beta[b, i, h] * r) - before @ dr
                d = d - np.outer(kk, dr)
                a = np.exp(g[b, i, h])
                dg[b, i, h] = np.sum(d * before)
                dS[b, h] = a * d if a != 0 else np.zeros_like(d)
    return dq, dk, dv, dg, db, dS


def top_logits(z, top):
    z = np.asarray(z, np.float64)
    index = np.full((z.shape[0], top), -1, np.int32)
    value = np.full((z.shape[0], top), -np.inf)
    for n, row in enumerate(z):
        ok = np.flatnonzero(row > -np.inf)                   # NaN compares false
        order = ok[np.argsort(-row[ok], kind="stable")][:top]
        index[n, :len(order)] = order
        value[n, :len(order)] = row[order]
    return index, value


def distill(z, index, value, temp, weight=None):
    """loss, log-sum-exp and the gradient of the sum of losses."""
    z, value = np.asarray(z, np.float64), np.asarray(value, np.float64)
    n, vocab = z.shape
    loss, lse, grad = np.zeros(n), np.zeros(n), np.zeros((n, vocab))
    for i in range(n):
        w = 1.0 if weight is None else float(weight[i])
        ok = (index[i] >= 0) & (index[i] < vocab) & (value[i] != -np.inf)
        if w == 0 or not ok.any():
            continue
        at, y = index[i][ok], value[i][ok] / temp
        p = np.exp(y - y.max())
        log_p = y - y.max() - np.log(p.sum())
        p = p / p.sum()
        x = z[i] / temp
        m = x.max()
        if m == -np.inf:
            lse[i], q = -np.inf, np.zeros(vocab)
            loss[i] = np.inf if (p > 0).any() else 0.0
        else:
            e = np.exp(x - m)
            lse[i], q = m + np.log(e.sum()), e / e.sum()
            on = p > 0
            log_q = (x[at[on]] - m) - np.log(e.sum())        # not x - lse: m may be the lowest value there is
            loss[i] = w * temp ** 2 * np.sum(p[on] * (log_p[on] - log_q))
        target = np.zeros(vocab)
        np.add.at(target, at, p)
        grad[i] = w * temp * (q - target)
    return loss, lse, grad
