"""What is timed of the operators around a student's memory: the embeddings of its tokens, the norms before and after a
block with its gate and residual sum, and the gated feed-forward block.

  embed      pql_embed_forward; with train, pql_embed_backward too: the table's gradient
  residual   pql_residual_forward; with train, pql_residual_backward too: every gradient
  ffn        pql_ffn_forward; with train, pql_ffn_backward too: every gradient (with keep from what the forward call
             has saved, without from the inputs alone)

The plain forms are elementary torch operations in 32 bits with gradients by torch's automatic differentiation, `exact`
the definitions in 64 bits with gradients written out.
"""
from __future__ import annotations

import math

import torch

own = False
DEVICE = "cuda:0"
EPS = 1e-5


def _embed(name, batch, steps, per_row, vocab, dim, dtype, train, ragged=False):
    return _named(name, dict(kind="embed", batch=batch, steps=steps, per_row=per_row, vocab=vocab, dim=dim, dtype=dtype,
                             train=train, ragged=ragged))


def _residual(name, batch, steps, dim, groups, dtype, train, form, gate="full", act="sigmoid", ragged=False):
    return _named(name, dict(kind="residual", batch=batch, steps=steps, dim=dim, groups=groups, dtype=dtype, train=train,
                             form=form, gate=gate, act=act, ragged=ragged))


def _ffn(name, batch, steps, dim, hidden, dtype, train, act="silu", keep=True, ragged=False, packed=False):
    return _named(name, dict(kind="ffn", batch=batch, steps=steps, dim=dim, hidden=hidden, dtype=dtype, train=train,
                             act=act, keep=keep, ragged=ragged, packed=packed))


def _named(name, c):
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # the Actor's step of the smallest program, 64 environments, 8 action dimensions of 51 bins: latency
        _embed("embed_step_64", 64, 1, 8, 8 * 51, 256, "float32", False),
        # the learner's step over short windows, 20 action dimensions of 51 bins: few tokens, each of them often
        _embed("embed_train_bins", 512, 32, 20, 20 * 51, 256, "float32", True, ragged=True),
        # the learner's step over long sequences of one token each from a large vocabulary: most rows of the gradient are zeros
        _embed("embed_train_vocab", 4, 2048, 1, 65536, 2048, "bfloat16", True),
        # the Actor's step of 16384 environments: after one block and before the next
        _residual("residual_step_16384", 16384, 1, 1024, 1, "bfloat16", False, "both"),
        # the learner's step over long sequences
        _residual("residual_train_sequences", 4, 2048, 2048, 1, "bfloat16", True, "both", ragged=True),
        # what stands behind a memory of 6 heads of 100: a norm for each head and its gate; rows on no 16-byte boundary
        _residual("residual_train_heads", 5, 333, 600, 6, "float32", True, "after", act="silu", ragged=True),
        # the step of 64 environments: latency
        _ffn("ffn_step_64", 64, 1, 256, 1024, "float32", False),
        # one token through a large block: its weights are read once
        _ffn("ffn_step_1", 1, 1, 4096, 16384, "bfloat16", False),
        # the Actor's step of 16384 environments
        _ffn("ffn_step_16384", 16384, 1, 512, 2048, "bfloat16", False, act="gelu"),
        # the learner's step over short windows, the framework's own 32-bit values
        _ffn("ffn_train_windows", 512, 32, 256, 1024, "float32", True, ragged=True),
        # the learner's step over long sequences, 16-bit values
        _ffn("ffn_train_sequences", 4, 2048, 2048, 8192, "bfloat16", True),
        # widths and lengths that fit no tile, tokens that are part of wider rows, nothing kept between the calls
        _ffn("ffn_train_ragged", 5, 333, 203, 677, "float32", True, act="gelu", keep=False, ragged=True, packed=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = [work(c) for c in listed()]
    bytes_, flops = max(m["bytes"] for m in most), max(m["flops"] for m in most)
    while True:
        kind = rng.choice(["embed", "residual", "ffn"])
        dtype, train = rng.choice(["float32", "bfloat16"]), rng.random() < 0.6
        steps = rng.choice([1, _log(rng, 1, 2048)])
        batch = _log(rng, 1, max(1, 16384 // steps))
        ragged = rng.random() < 0.4
        width = lambda lo, hi: rng.choice([8 * max(1, _log(rng, lo, hi) // 8), _log(rng, lo, hi)])  # noqa: E731
        if kind == "embed":
            c = _embed(None, batch, steps, rng.choice([1, 1, rng.randint(2, 24)]), _log(rng, 51, 65536), width(16, 2048),
                       dtype, train, ragged)
        elif kind == "residual":
            groups = rng.choice([1, 1, rng.randint(2, 16)])
            dim = width(32, 4096 // groups) * groups
            c = _residual(None, batch, steps, dim, groups, dtype, train, rng.choice(["both", "both", "before", "after"]),
                          rng.choice(["full", "full", "part", "none"]), rng.choice(["sigmoid", "silu"]), ragged)
        else:
            c = _ffn(None, batch, steps, width(32, 4096), width(64, 16384), dtype, train, rng.choice(["silu", "gelu", "relu"]),
                     rng.random() < 0.6, ragged, rng.random() < 0.2)
        w = work(c)
        # the lower bound leaves out only what is over in less time than a launch takes
        if 1e4 <= w["bytes"] <= bytes_ and w["flops"] <= flops and _plain_bytes(c) < 30e9:
            return c


def _plain_bytes(c):
    """Device memory the plain and the 64-bit forms take, about."""
    rows = c["batch"] * c["steps"]
    if c["kind"] == "embed":
        return 8.0 * c["dim"] * (2 * rows * c["per_row"] + 4 * rows + 2 * c["vocab"])
    if c["kind"] == "residual":
        return 8.0 * 24 * rows * c["dim"]
    return 8.0 * (8 * rows * (c["dim"] + c["hidden"]) + 9 * c["dim"] * c["hidden"])


def _lengths(c):
    """Lengths of a ragged batch: all between 0 and steps, the first ones full, empty and of one token."""
    n, t = c["batch"], c["steps"]
    out = [(t * ((7 * i) % 11) + 9) // 10 for i in range(n)]
    for i, x in enumerate((t, 0, 1)):
        if i < n:
            out[i] = x
    return [min(t, x) for x in out]


def work(c):
    size = 4 if c["dtype"] == "float32" else 2
    rows = sum(_lengths(c)) if c["ragged"] else c["batch"] * c["steps"]
    dim = c["dim"]
    if c["kind"] == "embed":
        read = min(rows * c["per_row"], c["vocab"])
        w = {"bytes": rows * (dim * size + 4 * c["per_row"]) + read * dim * size, "flops": float(rows * c["per_row"] * dim)}
        if c["train"]:              # the output's gradient in, the table's out
            w = {"bytes": w["bytes"] + (rows + c["vocab"]) * dim * size + 4 * rows * c["per_row"], "flops": 2 * w["flops"]}
        return w
    if c["kind"] == "residual":
        gate = {"full": dim, "part": c["groups"], "none": 0}[c["gate"] if c["form"] != "before" else "none"]
        x, y, u = c["form"] != "after", c["form"] != "before", c["form"] != "after"
        out = dim + dim * u
        one = rows * (dim * x + dim * y + gate + out) * size
        if not c["train"]:
            return {"bytes": one, "flops": 12.0 * rows * dim}
        return {"bytes": one + rows * (out + 2 * (dim * x + dim * y + gate)) * size, "flops": 40.0 * rows * dim}
    one, weights = rows * dim * size, 3 * dim * c["hidden"] * size
    if c["train"]:
        return {"bytes": 4 * one + 2 * weights, "flops": 18.0 * rows * dim * c["hidden"]}
    return {"bytes": 2 * one + weights, "flops": 6.0 * rows * dim * c["hidden"]}


# ---- inputs -------------------------------------------------------------------------------------
def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(int(seed) & 0x7FFFFFFF)
    s = {"embed": _prepare_embed, "residual": _prepare_residual, "ffn": _prepare_ffn}[c["kind"]](c, gen)
    s["case"] = c
    s["lengths"] = torch.tensor(_lengths(c), dtype=torch.int32, device=DEVICE) if c["ragged"] else None
    if own:
        s["held"] = _held(s)
    return s


def _normal(gen, dtype, *shape, by=1.0):
    return torch.randn(shape, generator=gen, device=DEVICE).mul_(by).to(getattr(torch, dtype))


def _prepare_embed(c, gen):
    n, t, m, vocab = c["batch"], c["steps"], c["per_row"], c["vocab"]
    if m > 1:                       # one bin for each dimension, most of them near the middle
        bins = max(1, vocab // m)
        at = torch.randn((n, t, m), generator=gen, device=DEVICE).mul_(bins / 6).add_(bins / 2).floor_().clamp_(0, bins - 1)
        tokens = at + bins * torch.arange(m, device=DEVICE)
    else:                           # few tokens that are frequent, many that are rare
        tokens = (vocab * torch.rand((n, t, m), generator=gen, device=DEVICE) ** 4).floor_().clamp_(0, vocab - 1)
    # what has no token: the first step of an episode has no last answer
    none = torch.rand((n, t, 1), generator=gen, device=DEVICE) < 0.01
    s = dict(tokens=tokens.masked_fill(none, -1).to(torch.int32), table=_normal(gen, c["dtype"], vocab, c["dim"]), scale=c["dim"] ** 0.5)
    if c["train"]:
        s["out_grad"] = _normal(gen, c["dtype"], n, t, c["dim"])
    return s


def _prepare_residual(c, gen):
    n, t, d, dt = c["batch"], c["steps"], c["dim"], c["dtype"]
    s = dict(x=None, y=None, gate=None, post=None, pre=None, next_grad=None)
    if c["form"] != "after":
        s["x"] = _normal(gen, dt, n, t, d, by=2.0)
        s["pre"] = 1 + 0.2 * _normal(gen, "float32", d)
    if c["form"] != "before":
        s["y"] = _normal(gen, dt, n, t, d) * (0.5 + torch.rand((n, t, 1), generator=gen, device=DEVICE)).to(getattr(torch, dt))
        s["post"] = 0.5 + 0.2 * _normal(gen, "float32", d)
        if c["gate"] != "none":
            s["gate"] = _normal(gen, dt, n, t, d if c["gate"] == "full" else c["groups"])
    s["scale_x"], s["scale_y"] = 1.0, (0.5 if c["form"] == "both" else 1.0)
    if c["train"]:
        s["sum_grad"] = _normal(gen, dt, n, t, d)
        if c["form"] != "after":
            s["next_grad"] = _normal(gen, dt, n, t, d)
    return s


def _prepare_ffn(c, gen):
    n, t, d, f, dt = c["batch"], c["steps"], c["dim"], c["hidden"], c["dtype"]
    if c["packed"]:                 # some columns of wider rows
        x = _normal(gen, dt, n, t, d + 24)[..., 8:8 + d]
    else:
        x = _normal(gen, dt, n, t, d)
    s = dict(x=x, gate=_normal(gen, dt, f, d, by=d ** -0.5), up=_normal(gen, dt, f, d, by=d ** -0.5),
             down=_normal(gen, dt, d, f, by=f ** -0.5))
    if c["train"]:
        s["out_grad"] = _normal(gen, dt, n, t, d)
    return s


# ---- the framework's calls ------------------------------------------------------------------------
def _held(s):
    """What a program keeps between passes: a context, its buffers and the descriptions of them."""
    from paper_2307_12983_amd import block as K
    c, ctx = s["case"], K.BlockContext()
    h = dict(ctx=ctx)
    rows = lambda t: None if t is None else K.Rows(t)  # noqa: E731
    like = lambda t: None if t is None else torch.empty(t.shape, dtype=t.dtype, device=DEVICE)  # noqa: E731
    new = lambda *shape: torch.empty(shape, dtype=getattr(torch, c["dtype"]), device=DEVICE)  # noqa: E731
    n, t, d = c["batch"], c["steps"], c["dim"]
    if c["kind"] == "embed":
        h["shape"] = K.embed_shape(s["tokens"], s["table"], s["scale"])
        h["table"] = K.Rows(s["table"])
        h["out"] = new(n, t, d)
        h["out_d"] = K.Rows(h["out"])
        if c["train"]:
            h["out_grad_d"] = K.Rows(s["out_grad"])
            h["grad"] = like(s["table"])
            h["grad_d"] = K.Rows(h["grad"])
            h["work"] = K.workspace(ctx.embed_workspace_bytes(h["shape"]), DEVICE)
    elif c["kind"] == "residual":
        gate = s["gate"]
        h["shape"] = K.residual_shape(n, t, d, getattr(torch, c["dtype"]), groups=c["groups"],
                                      gate_cols=0 if gate is None else gate.shape[-1], gate_act=c["act"],
                                      eps_post=EPS if s["y"] is not None else 0.0, eps_pre=EPS if s["x"] is not None else 0.0,
                                      scale_x=s["scale_x"], scale_y=s["scale_y"])
        h["input"] = K.ResidualInput(h["shape"], s["x"], s["y"], gate, s["post"], s["pre"], s["lengths"])
        h["sum"], h["next"] = new(n, t, d), (new(n, t, d) if s["x"] is not None else None)
        h["sum_d"], h["next_d"] = rows(h["sum"]), rows(h["next"])
        if c["train"]:
            h["grad"] = {k: like(s[k]) for k in ("x", "y", "gate", "post", "pre")}
            h["grad_d"] = K.ResidualGrad(h["shape"], **h["grad"])
            h["sum_grad_d"], h["next_grad_d"] = rows(s["sum_grad"]), rows(s["next_grad"])
            h["work"] = K.workspace(ctx.residual_workspace_bytes(h["shape"]), DEVICE)
    else:
        h["shape"] = K.ffn_shape(s["x"], s["gate"], c["act"])
        h["input"] = K.FfnInput(h["shape"], s["x"], s["gate"], s["up"], s["down"], s["lengths"])
        h["out"] = new(n, t, d)
        h["out_d"] = K.Rows(h["out"])
        h["saved"] = K.workspace(ctx.ffn_saved_bytes(h["shape"]), DEVICE) if c["train"] and c["keep"] else None
        need = ctx.ffn_workspace_bytes(h["shape"], K.FFN_FORWARD)
        if c["train"]:
            need = max(need, ctx.ffn_workspace_bytes(h["shape"], K.FFN_BACKWARD if c["keep"] else K.FFN_BACKWARD_ALONE))
            h["grad"] = {k: like(s[k]) for k in ("x", "gate", "up", "down")}
            h["grad_d"] = K.FfnGrad(h["shape"], **h["grad"])
            h["out_grad_d"] = K.Rows(s["out_grad"])
        h["work"] = K.workspace(need, DEVICE)
    return h


def _run_own(s):
    c, h = s["case"], s["held"]
    ctx = h["ctx"]
    if c["kind"] == "embed":
        ctx.pql_embed_forward(h["shape"], s["tokens"], s["lengths"], h["table"], h["out_d"])
        r = dict(out=h["out"])
        if c["train"]:
            ctx.pql_embed_backward(h["shape"], s["tokens"], s["lengths"], h["out_grad_d"], h["grad_d"], h["work"])
            r["dtable"] = h["grad"]
    elif c["kind"] == "residual":
        ctx.pql_residual_forward(h["shape"], h["input"], h["sum_d"], h["next_d"])
        r = dict(sum=h["sum"], next=h["next"])
        if c["train"]:
            ctx.pql_residual_backward(h["shape"], h["input"], h["sum_grad_d"], h["next_grad_d"], h["grad_d"], h["work"])
            r.update({"d" + k: x for k, x in h["grad"].items()})
    else:
        ctx.pql_ffn_forward(h["shape"], h["input"], h["out_d"], h["saved"], h["work"])
        r = dict(out=h["out"])
        if c["train"]:
            ctx.pql_ffn_backward(h["shape"], h["input"], h["saved"], h["out_grad_d"], h["grad_d"], h["work"])
            r.update({"d" + k: x for k, x in h["grad"].items()})
    return {k: x for k, x in r.items() if x is not None}


# ---- plain forms ----------------------------------------------------------------------------------
def run(s):
    if own:
        return _run_own(s)
    c = s["case"]
    f = {"embed": _plain_embed, "residual": _plain_residual, "ffn": _plain_ffn}[c["kind"]]
    if not c["train"]:
        with torch.no_grad():
            return {k: x.to(s[_LIKE[c["kind"]](s)].dtype) for k, x in f(s, s).items()}
    names = [k for k in ("x", "y", "gate", "up", "down", "post", "pre", "table") if s.get(k) is not None]
    x = {**s, **{k: s[k].float().requires_grad_() for k in names}}
    out = f(s, x)
    given = {"out": "out_grad", "sum": "sum_grad", "next": "next_grad"}
    grads = torch.autograd.grad(list(out.values()), [x[k] for k in names], [s[given[k]].float() for k in out])
    dt = s[_LIKE[c["kind"]](s)].dtype
    r = {k: v.detach().to(dt) for k, v in out.items()}
    r.update({"d" + k: g.to(s[k].dtype) for k, g in zip(names, grads)})
    return r


# whose type a kind's outputs have
_LIKE = {"embed": lambda s: "table", "residual": lambda s: "x" if s["x"] is not None else "y", "ffn": lambda s: "x"}


def _counted(s):
    """Which tokens count, [batch, steps, 1]; None for all."""
    c = s["case"]
    if s["lengths"] is None:
        return None
    return (torch.arange(c["steps"], device=DEVICE)[None] < s["lengths"][:, None])[..., None]


def _only(s, x):
    real = _counted(s)
    return x if real is None else torch.where(real, x, 0.0)


def _act(name, x):
    if name == "sigmoid":
        return torch.sigmoid(x)
    if name == "silu":
        return x * torch.sigmoid(x)
    if name == "gelu":
        return 0.5 * x * (1 + torch.erf(x * 0.5 ** 0.5))
    return torch.clamp(x, min=0)


def _plain_embed(s, x):
    tokens = s["tokens"].long()
    there = (tokens >= 0) & (tokens < s["case"]["vocab"])
    rows = x["table"].float()[tokens.clamp(0, s["case"]["vocab"] - 1)]
    return dict(out=_only(s, s["scale"] * torch.where(there[..., None], rows, 0.0).sum(2)))


def _plain_residual(s, x):
    c = s["case"]
    total = None
    if x["x"] is not None:
        total = s["scale_x"] * x["x"].float()
    if x["y"] is not None:
        y = x["y"].float().unflatten(-1, (c["groups"], -1))
        y = (y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS)).flatten(-2) * x["post"]
        if x["gate"] is not None:
            g = _act(c["act"], x["gate"].float())
            y = y * (g if c["gate"] == "full" else g.repeat_interleave(c["dim"] // c["groups"], -1))
        total = s["scale_y"] * y if total is None else total + s["scale_y"] * y
    out = dict(sum=_only(s, total))
    if x["x"] is not None:
        out["next"] = _only(s, x["pre"] * total * torch.rsqrt((total * total).mean(-1, keepdim=True) + EPS))
    return out


def _plain_ffn(s, x):
    v = _only(s, x["x"].float())
    a, b = torch.matmul(v, x["gate"].float().T), torch.matmul(v, x["up"].float().T)
    return dict(out=_only(s, torch.matmul(_act(s["case"]["act"], a) * b, x["down"].float().T)))


# ---- 64 bits ----------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    c = s["case"]
    if c["ragged"]:
        on = (torch.arange(c["steps"], device=DEVICE)[None] < s["lengths"][:, None]).reshape(-1)
    else:
        on = torch.ones(c["batch"] * c["steps"], dtype=torch.bool, device=DEVICE)
    return {"embed": _exact_embed, "residual": _exact_residual, "ffn": _exact_ffn}[c["kind"]](c, s, on)


def _live(x, on):
    """The rows that count, in 64 bits."""
    return None if x is None else x.reshape(on.numel(), -1)[on].double()


def _spread(c, x, on):
    out = torch.zeros((on.numel(), x.shape[1]), dtype=torch.float64, device=DEVICE)
    out[on] = x
    return out.reshape(c["batch"], c["steps"], -1)


def _exact_embed(c, s, on):
    tokens, table = s["tokens"].reshape(on.numel(), -1)[on].long(), s["table"].double()
    out = torch.zeros((tokens.shape[0], c["dim"]), dtype=torch.float64, device=DEVICE)
    grad = torch.zeros_like(table)
    for j in range(c["per_row"]):
        at = torch.nonzero(tokens[:, j] >= 0)[:, 0]
        out[at] += s["scale"] * table[tokens[at, j]]
        if c["train"]:
            grad.index_put_((tokens[at, j],), s["scale"] * _live(s["out_grad"], on)[at], accumulate=True)
    r = dict(out=_spread(c, out, on))
    if c["train"]:
        r["dtable"] = grad
    return r


def _exact_residual(c, s, on):
    x, y, gate = _live(s["x"], on), _live(s["y"], on), _live(s["gate"], on)
    rows, d, groups = int(on.sum()), c["dim"], c["groups"]
    wide = lambda g: g if g.shape[1] == d else g[:, :, None].expand(rows, groups, d // groups).reshape(rows, d)  # noqa: E731
    total = torch.zeros((rows, d), dtype=torch.float64, device=DEVICE)
    if x is not None:
        total += s["scale_x"] * x
    if y is not None:
        parts = y.reshape(rows, groups, -1)
        size = torch.sqrt((parts ** 2).mean(2, keepdim=True) + EPS)
        unit = (parts / size).reshape(rows, d)
        post = s["post"].double()
        opened, slope = torch.ones_like(unit), None
        if gate is not None:
            g = wide(gate)
            sig = 1 / (1 + torch.exp(-g))
            opened, slope = (sig, sig * (1 - sig)) if c["act"] == "sigmoid" else (g * sig, sig * (1 + g * (1 - sig)))
        total += s["scale_y"] * opened * post * unit
    r = dict(sum=_spread(c, total, on))
    dtotal = _live(s["sum_grad"], on) if c["train"] else None
    if x is not None:
        pre = s["pre"].double()
        norm = torch.sqrt((total ** 2).mean(1, keepdim=True) + EPS)
        r["next"] = _spread(c, pre * total / norm, on)
        if c["train"]:
            du = _live(s["next_grad"], on)
            hat = total / norm
            r["dpre"] = (du * hat).sum(0)
            dhat = du * pre
            dtotal = dtotal + (dhat - hat * (dhat * hat).mean(1, keepdim=True)) / norm
            r["dx"] = _spread(c, s["scale_x"] * dtotal, on)
    if c["train"] and y is not None:
        dz = s["scale_y"] * dtotal
        r["dpost"] = (dz * opened * unit).sum(0)
        if gate is not None:
            dgate = dz * post * unit * slope
            r["dgate"] = _spread(c, dgate if gate.shape[1] == d else dgate.reshape(rows, groups, -1).sum(2), on)
        dunit = (dz * opened * post).reshape(rows, groups, -1)
        u = unit.reshape(rows, groups, -1)
        r["dy"] = _spread(c, ((dunit - u * (dunit * u).mean(2, keepdim=True)) / size).reshape(rows, d), on)
    return r


def _exact_ffn(c, s, on):
    x, gate, up, down = _live(s["x"], on), s["gate"].double(), s["up"].double(), s["down"].double()
    a, b = x @ gate.t(), x @ up.t()
    if c["act"] == "silu":
        sig = 1 / (1 + torch.exp(-a))
        act, slope = a * sig, sig * (1 + a * (1 - sig))
    elif c["act"] == "gelu":
        half = 0.5 * torch.special.erfc(-a / math.sqrt(2.0))
        act, slope = a * half, half + a * torch.exp(-0.5 * a * a) / math.sqrt(2 * math.pi)
    else:
        act, slope = torch.where(a > 0, a, 0.0), (a > 0).double()
    r = dict(out=_spread(c, (act * b) @ down.t(), on))
    if c["train"]:
        do = _live(s["out_grad"], on)
        dm = do @ down
        da, db = dm * b * slope, dm * act
        r.update(dx=_spread(c, da @ gate + db @ up, on), dgate=da.t() @ x, dup=db.t() @ x, ddown=do.t() @ (act * b))
    return r
