"""Double-precision reference of the operators around a student's memory (test infrastructure only).

Rows are arrays [batch, steps, columns]; `lengths` (a list or None) says how many steps of each sequence count.  What does
not count is zero in every result and has no part in the gradients of weights.  Gradients are written out by hand; they
are checked against differences in tests/test_block_host.py.
"""
import math

import numpy as np


def counted(shape, lengths):
    n, t = shape
    if lengths is None:
        return np.ones((n, t), bool)
    return np.arange(t)[None] < np.clip(np.asarray(lengths), 0, t)[:, None]


def only(x, real):
    return np.where(real[..., None], x, 0.0)


# ---- embeddings -------------------------------------------------------------------------------------
def embed(tokens, table, scale, lengths=None):
    tokens = np.asarray(tokens)
    real = counted(tokens.shape[:2], lengths)
    there = (tokens >= 0) & (tokens < len(table)) & real[..., None]
    rows = np.where(there[..., None], table[np.where(there, tokens, 0)], 0.0)
    return scale * rows.sum(2)


def embed_grad(tokens, vocab, scale, out_grad, lengths=None):
    tokens = np.asarray(tokens)
    real = counted(tokens.shape[:2], lengths)
    grad = np.zeros((vocab, out_grad.shape[-1]))
    for b, t, j in np.argwhere((tokens >= 0) & (tokens < vocab) & real[..., None]):
        grad[tokens[b, t, j]] += scale * out_grad[b, t]
    return grad


# ---- activations --------------------------------------------------------------------------------------
_erf = np.vectorize(math.erf, otypes=[float])


def activate(act, x):
    """The function and its derivative."""
    if act == "none":
        return x, np.ones_like(x)
    if act == "relu":
        return np.where(x > 0, x, 0.0), np.where(x > 0, 1.0, 0.0)
    if act == "gelu":
        half = 0.5 * (1 + _erf(x / math.sqrt(2)))
        return x * half, half + x * np.exp(-0.5 * x * x) / math.sqrt(2 * math.pi)
    e = np.exp(-np.abs(x))                              # s and 1 - s, neither from the other
    s, rest = np.where(x < 0, e, 1.0) / (1 + e), np.where(x < 0, 1.0, e) / (1 + e)
    return (s, s * rest) if act == "sigmoid" else (x * s, s * (1 + x * rest))


# ---- norms, gate and residual sum -----------------------------------------------------------------------
class Residual:
    """sum = ax x + ay act(gate) post N(y), next = pre N(sum); parts of None are left out, an eps of 0 is no norm."""

    def __init__(self, x, y, gate, post, pre, groups=1, act="none", eps_post=0.0, eps_pre=0.0, scale_x=1.0, scale_y=1.0, lengths=None):
        like = x if x is not None else y
        n, t, d = like.shape
        self.real = real = counted((n, t), lengths)
        clean = lambda z: None if z is None else only(z, real)  # noqa: E731
        x, y, gate = clean(x), clean(y), clean(gate)
        self.x, self.y, self.groups, self.d, self.scale_x, self.scale_y = x, y, groups, d, scale_x, scale_y
        self.post = np.ones(d) if post is None else post
        self.pre = np.ones(d) if pre is None else pre
        self.gate_cols = 0 if gate is None else gate.shape[-1]
        total = np.zeros((n, t, d))
        if x is not None:
            total = total + scale_x * x
        self.eps_post, self.eps_pre = eps_post, eps_pre
        if y is not None:
            parts = y.reshape(n, t, groups, -1)
            self.r = 1 / np.sqrt((parts ** 2).mean(-1, keepdims=True) + eps_post) if eps_post else np.ones((n, t, groups, 1))
            self.unit = (parts * self.r).reshape(n, t, d)
            if gate is None:
                self.open, self.slope = np.ones((n, t, d)), np.zeros((n, t, d))
            else:
                wide = gate if gate.shape[-1] == d else np.repeat(gate, d // groups, axis=-1)
                self.open, self.slope = activate(act, wide)
            total = total + scale_y * self.open * self.post * self.unit
        self.total = total
        self.f = 1 / np.sqrt((total ** 2).mean(-1, keepdims=True) + eps_pre) if eps_pre else np.ones((n, t, 1))
        self.sum, self.next = only(total, real), only(self.pre * total * self.f, real)

    def grad(self, sum_grad, next_grad):
        n, t, d = self.total.shape
        real = self.real
        dh = np.zeros((n, t, d)) if sum_grad is None else only(sum_grad, real)
        r = dict(x=None, y=None, gate=None, post=None, pre=None)
        if next_grad is not None:
            du, hat = only(next_grad, real), self.total * self.f
            r["pre"] = (du * hat).sum((0, 1))
            dhat = du * self.pre
            dh = dh + self.f * (dhat - (hat * (dhat * hat).mean(-1, keepdims=True) if self.eps_pre else 0.0))
        dh = only(dh, real)
        if self.x is not None:
            r["x"] = self.scale_x * dh
        if self.y is not None:
            dz = self.scale_y * dh
            r["post"] = (dz * self.open * self.unit).sum((0, 1))
            if self.gate_cols:
                g = only(dz * self.post * self.unit * self.slope, real)
                r["gate"] = g if self.gate_cols == d else g.reshape(n, t, self.groups, -1).sum(-1)
            dn, u = (dz * self.open * self.post).reshape(n, t, self.groups, -1), self.unit.reshape(n, t, self.groups, -1)
            dy = self.r * (dn - (u * (dn * u).mean(-1, keepdims=True) if self.eps_post else 0.0))
            r["y"] = only(dy.reshape(n, t, d), real)
        return r


# ---- gated feed-forward block ----------------------------------------------------------------------------
def ffn(x, gate, up, down, act, lengths=None):
    x = only(x, counted(x.shape[:2], lengths))
    return (activate(act, x @ gate.T)[0] * (x @ up.T)) @ down.T


def ffn_grad(x, gate, up, down, act, out_grad, lengths=None):
    real = counted(x.shape[:2], lengths)
    x, out_grad = only(x, real), only(out_grad, real)
    a, b = x @ gate.T, x @ up.T
    f, slope = activate(act, a)
    dm = out_grad @ down
    da, db = dm * b * slope, dm * f
    flat = lambda z: z.reshape(-1, z.shape[-1])  # noqa: E731
    return dict(x=da @ gate + db @ up, gate=flat(da).T @ flat(x), up=flat(db).T @ flat(x), down=flat(out_grad).T @ flat(f * b))
