"""The operators around a student's memory on the GPU against the double-precision reference.

Tolerances, from the arithmetic (u = 2^-24, the rounding of a 32-bit operation):
  embeddings   a sum of k terms and a factor: relative to the sum of the terms' sizes at most (k + 1) u, taken element by element.
  residual     a mean over d squares and some ten operations: 2-norm within (sqrt(d) / 2 + 20) u of the result's, d at most 8192:
               4e-6.  Weights' gradients are sums over rows of such terms, each sum rounded at most `rows` times, at random: the
               same bound with the rows' number in the place of d, at the size of the terms.
  ffn          products over K elements of terms with an error of u each, accumulated in 32 bits: (sqrt(K) + 10) u of the 2-norm
               for each of at most three products in a row; K at most 16384: 3 * 138 u = 2.5e-5.  In bf16 what lies between
               two products (m, da, db) is rounded to bf16 once: 2^-8 / sqrt 3 / 2 = 1.2e-3 of its 2-norm at most, which the next
               product passes on to a result whose terms have random signs as it is, or up to twice that where one factor is smooth.
An output in bf16 is rounded once more, by at most half the spacing of its values, which is taken off first.  Single elements
may be off by 40 times the bound of the norm, relative to the larger of the element and the root mean square.  """
import math

import numpy as np
import pytest

from oracle import block_oracle as O

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def env():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible: the gpu-marked tests need a real MI355X")
    from paper_2307_12983_amd import block as K
    return torch, K, K.BlockContext()


def error_of(got, want):
    """Absolute errors beyond the rounding of the output's type; both hold the same values that are not finite."""
    bf16 = str(got.dtype) == "torch.bfloat16"
    got, want = got.detach().double().cpu().numpy(), np.asarray(want, np.float64)
    assert got.shape == want.shape
    assert np.all(np.isfinite(got)) and np.all(np.isfinite(want))
    off = np.abs(got - want)
    if bf16:                                            # 8 significant bits: half a spacing is 2^(exponent - 8)
        size = np.maximum(np.abs(got), np.abs(want))
        off = np.maximum(0.0, off - np.exp2(np.floor(np.log2(np.maximum(size, 1e-37))) - 8))
    return off, want


def close(got, want, what, bound):
    off, want = error_of(got, want)
    norm = np.linalg.norm(want)
    err = np.linalg.norm(off)
    assert err <= bound * norm, "%s: error %.3g of the norm, %.3g allowed" % (what, err / norm if norm else np.inf, bound)
    if norm:
        worst = np.max(off / np.maximum(norm / np.sqrt(want.size), np.abs(want)))
        assert worst <= 40 * bound, "%s: an element off by %.3g" % (what, worst)


class Made:
    """Tensors in a layout, kept with their values in double precision."""

    def __init__(self, env, seed, dtype, layout="dense", lengths=None):
        self.torch = env[0]
        self.rng, self.dt, self.layout, self.lengths = np.random.default_rng(seed), getattr(env[0], dtype), layout, lengths

    def place(self, values, shape=None):
        """Rows of those values; what does not count is poisoned."""
        torch = self.torch
        v = np.array(values, np.float64)
        if self.lengths is not None and v.ndim == 3:
            v[~O.counted(v.shape[:2], self.lengths)] = np.nan
        t = torch.tensor(v).to(self.dt).cuda()
        if self.layout == "offset":                     # rows on no 16-byte boundary, something else between them
            big = torch.full((*t.shape[:-1], t.shape[-1] + 3), float("nan"), dtype=t.dtype, device="cuda")
            big[..., 1:1 + t.shape[-1]] = t
            t = big[..., 1:1 + t.shape[-1]]
        elif self.layout == "wide":                     # aligned rows, something else between them
            big = torch.full((*t.shape[:-1], t.shape[-1] + 24), float("nan"), dtype=t.dtype, device="cuda")
            big[..., 8:8 + t.shape[-1]] = t
            t = big[..., 8:8 + t.shape[-1]]
        return t

    def normal(self, *shape, by=1.0):
        return self.place(by * self.rng.standard_normal(shape))

    def out(self, *shape):
        return self.place(np.full(shape, 7.0))

    def host(self, t):
        return None if t is None else t.double().cpu().numpy()


def lengths_of(torch, lengths):
    return None if lengths is None else torch.tensor(lengths, dtype=torch.int32).cuda()


def label(c):
    return "-".join(str(v).replace(" ", "")[:40] for v in (c.values() if isinstance(c, dict) else c))


# ---- embeddings -----------------------------------------------------------------------------------------
EMBED = [
    # batch, steps, per_row, vocab, dim, dtype, layout, lengths, tokens
    (1, 1, 1, 1, 1, "float32", "dense", None, "any"),
    (1, 1, 3, 7, 64, "bfloat16", "dense", None, "any"),
    (64, 1, 8, 408, 256, "float32", "dense", None, "any"),
    (5, 33, 20, 1020, 72, "bfloat16", "dense", [33, 0, 1, 12, 40], "any"),
    (3, 70, 1, 50, 100, "float32", "offset", [70, -3, 69], "any"),
    (4, 64, 2, 300, 513, "bfloat16", "offset", None, "any"),
    (2, 40, 5, 9, 1024, "float32", "wide", None, "any"),
    (8, 100, 1, 5, 40, "float32", "dense", None, "equal"),              # one token everywhere
    (6, 50, 1, 100000, 24, "bfloat16", "dense", None, "any"),           # few of many
    (2, 31, 1, 40, 16, "float32", "dense", None, "none"),               # no token at all
    (2, 31, 1, 40, 16, "float32", "dense", [0, 0], "any"),              # nothing that counts
    (40, 256, 1, 1000, 32, "float32", "dense", None, "any"),            # more places than are sorted in one launch
    (40, 256, 1, 1023, 32, "float32", "dense", None, "any"),            # keys of ten bits and the one beyond them
    (40, 256, 1, 1024, 32, "float32", "dense", None, "any"),
    (40, 64, 4, 70000, 8, "bfloat16", "dense", list(range(40)), "any"),
    (40, 256, 2, 2000000, 4, "float32", "dense", None, "far"),          # three digits
    (64, 512, 1, 300, 8, "float32", "dense", None, "equal"),
    (300, 512, 1, 64, 12, "float32", "dense", None, "any"),             # chunks of more than 32 places
]


def embed_inputs(env, case, seed=0):
    torch = env[0]
    n, t, m, vocab, dim, dtype, layout, lengths, which = case
    made = Made(env, seed, dtype, layout, None)
    tokens = made.rng.integers(-1, vocab + 1, (n, t, m))                # the ends are no tokens
    if which == "equal":
        tokens[:] = vocab // 2
    elif which == "none":
        tokens[:] = np.where(tokens % 2 == 0, -5, vocab + 3)
    elif which == "far":
        tokens = vocab - 1 - tokens % 100
    table = made.normal(vocab, dim)
    made.lengths = lengths
    return made, torch.tensor(tokens, dtype=torch.int32).cuda(), tokens, table, made.normal(n, t, dim), lengths_of(torch, lengths)


@pytest.mark.parametrize("case", EMBED, ids=label)
def test_embeddings_and_their_gradient(env, case):
    torch, K, ctx = env
    made, tokens, host, table, out_grad, lengths = embed_inputs(env, case)
    n, t, m, vocab, dim = case[:5]
    scale = float(np.float32(dim ** 0.5))
    shape = K.embed_shape(tokens, table, scale)
    out = made.out(n, t, dim)
    ctx.pql_embed_forward(shape, tokens, lengths, K.Rows(table), K.Rows(out))
    size = O.embed(host, np.abs(made.host(table)), scale, case[7])
    off, want = error_of(out, O.embed(host, made.host(table), scale, case[7]))
    assert np.all(off <= (m + 1) * U * size)
    made.lengths = None
    grad = made.out(vocab, dim)
    ctx.pql_embed_backward(shape, tokens, lengths, K.Rows(out_grad), K.Rows(grad), K.workspace(ctx.embed_workspace_bytes(shape)))
    clean = np.nan_to_num(made.host(out_grad))
    size, count = O.embed_grad(host, vocab, scale, np.abs(clean), case[7]), O.embed_grad(host, vocab, 1.0, np.ones((n, t, 1)), case[7])
    off, want = error_of(grad, O.embed_grad(host, vocab, scale, clean, case[7]))
    assert np.all(off <= (count + 1) * U * size)


def test_embedding_gradients_have_one_order(env):
    torch, K, ctx = env
    made, tokens, _, table, out_grad, _ = embed_inputs(env, (40, 256, 3, 200, 96, "float32", "dense", None, "any"))
    shape = K.embed_shape(tokens, table, 1.0)
    results = []
    for _ in range(3):
        grad, space = made.out(200, 96), K.workspace(ctx.embed_workspace_bytes(shape))
        space.random_(0, 255)
        ctx.pql_embed_backward(shape, tokens, None, K.Rows(out_grad), K.Rows(grad), space)
        results.append(grad)
    assert all(torch.equal(results[0], r) for r in results)


def test_embeddings_leave_what_is_not_theirs(env):
    """Neither the gaps between rows nor what lies behind the last one are written."""
    torch, K, ctx = env
    tokens = torch.randint(0, 30, (3, 5, 2), dtype=torch.int32, device="cuda")
    table, big, grad = torch.randn(30, 20, device="cuda"), torch.full((17, 28), 7.0, device="cuda"), torch.full((33, 28), 7.0, device="cuda")
    shape = K.embed_shape(tokens, table, 1.0)
    ctx.pql_embed_forward(shape, tokens, None, K.Rows(table), K.Rows(big[:15, 4:24]))
    ctx.pql_embed_backward(shape, tokens, None, K.Rows(big[:15, 4:24]), K.Rows(grad[:30, 4:24]), K.workspace(ctx.embed_workspace_bytes(shape)))
    for x, n in ((big, 15), (grad, 30)):
        assert bool((x[n:] == 7).all()) and bool((x[:, :4] == 7).all()) and bool((x[:, 24:] == 7).all())
        assert not bool((x[:n, 4:24] == 7).any())


# ---- norms, gate and residual sum --------------------------------------------------------------------------
def residual_case(batch, steps, dim, dtype, groups=1, form="both", gate="full", act="sigmoid", layout="dense", lengths=None, eps=(1e-5, 1e-5),
                  weights=True, scales=(1.0, 0.5)):
    return dict(locals())


# Parts of one element have an eps of their values' size: with a small one y / |y| hardly depends on y, and its gradient is what is
# left of two terms that cancel.
RESIDUAL = [
    residual_case(1, 1, 1, "float32", eps=(0.5, 0.5)),
    residual_case(1, 1, 8, "bfloat16"),
    residual_case(64, 1, 256, "float32"),
    residual_case(5, 33, 1024, "bfloat16", lengths=[33, 0, 1, 12, 40]),
    residual_case(3, 9, 2048, "bfloat16", act="silu"),
    residual_case(2, 5, 4096, "float32", act="gelu"),
    residual_case(2, 3, 8192, "float32"),
    residual_case(2, 3, 8191, "bfloat16", layout="offset"),
    residual_case(7, 11, 600, "float32", groups=6, form="after", act="silu", layout="offset", lengths=[11, 0, 1, 5, 9, -1, 99]),
    residual_case(7, 11, 600, "float32", groups=6, act="silu"),
    residual_case(3, 17, 512, "bfloat16", groups=4, gate="part", act="sigmoid", lengths=[17, 2, 9]),
    residual_case(3, 17, 512, "float32", groups=8, form="after", gate="part", act="none"),
    residual_case(9, 4, 72, "float32", groups=3, layout="wide"),
    residual_case(9, 4, 75, "bfloat16", groups=25, layout="offset", act="relu"),
    residual_case(2, 6, 256, "float32", groups=256, eps=(0.5, 1e-5)),
    residual_case(2, 6, 7936, "float32", groups=248),
    residual_case(2, 6, 2304, "bfloat16", groups=256),
    residual_case(1, 5, 8190, "float32", groups=2, form="after"),
    residual_case(4, 40, 128, "float32", form="before"),
    residual_case(4, 40, 128, "float32", eps=(0.0, 1e-5)),
    residual_case(4, 40, 128, "bfloat16", eps=(1e-5, 0.0), weights=False),
    residual_case(4, 40, 130, "float32", eps=(0.0, 0.0), gate="none", scales=(0.7, -1.5)),
    residual_case(300, 20, 64, "float32", scales=(1.0, 1.0)),
    residual_case(2000, 9, 24, "bfloat16", act="gelu"),
    residual_case(3, 1, 256, "float32", lengths=[0, 0, 0]),
]


class ResidualCall:
    def __init__(self, env, c, seed=0, by=1.0):
        torch, K, ctx = self.env = env
        self.c = c
        self.made = m = Made(env, seed, c["dtype"], c["layout"], c["lengths"])
        n, t, d = c["batch"], c["steps"], c["dim"]
        has_x, has_y = c["form"] != "after", c["form"] != "before"
        self.x = m.normal(n, t, d, by=2.0 * by) if has_x else None
        self.y = m.normal(n, t, d, by=by) if has_y else None
        cols = {"none": 0, "part": c["groups"], "full": d}[c["gate"] if has_y else "none"]
        self.gate = m.normal(n, t, cols) if cols else None
        weight = lambda: torch.tensor(1 + 0.3 * m.rng.standard_normal(d)).float().cuda()  # noqa: E731
        self.post = weight() if has_y and c["weights"] else None
        self.pre = weight() if has_x and c["weights"] else None
        self.sum_grad, self.next_grad = m.normal(n, t, d), m.normal(n, t, d) if has_x else None
        self.scales = [float(np.float32(x)) for x in c["scales"]]
        self.eps = [float(np.float32(x)) for x in c["eps"]]
        self.lengths = lengths_of(torch, c["lengths"])
        self.shape = K.residual_shape(n, t, d, self.made.dt, c["groups"], cols, c["act"], *self.eps, *self.scales)
        self.given = K.ResidualInput(self.shape, self.x, self.y, self.gate, self.post, self.pre, self.lengths)
        h = m.host
        self.want = O.Residual(h(self.x), h(self.y), h(self.gate), h(self.post), h(self.pre), c["groups"], c["act"], *self.eps, *self.scales, c["lengths"])

    def outs(self, clean=True):
        keep, self.made.lengths = self.made.lengths, None
        n, t, d = self.c["batch"], self.c["steps"], self.c["dim"]
        r = self.made.out(n, t, d), (self.made.out(n, t, d) if self.x is not None else None)
        self.made.lengths = keep
        return r

    def forward(self):
        _, K, ctx = self.env
        total, after = self.outs()
        ctx.pql_residual_forward(self.shape, self.given, K.Rows(total), None if after is None else K.Rows(after))
        return total, after

    def backward(self, leave=()):
        torch, K, ctx = self.env
        keep, self.made.lengths = self.made.lengths, None
        g = {k: None if getattr(self, k) is None or k in leave else self.made.out(*getattr(self, k).shape) for k in ("x", "y", "gate")}
        self.made.lengths = keep
        g.update({k: torch.full((self.c["dim"],), 7.0, device="cuda") if getattr(self, k) is not None and k not in leave else None for k in ("post", "pre")})
        if self.x is not None and self.pre is None and "pre" not in leave:
            g["pre"] = torch.full((self.c["dim"],), 7.0, device="cuda")
        rows = lambda t: None if t is None else K.Rows(t)  # noqa: E731
        ctx.pql_residual_backward(self.shape, self.given, rows(self.sum_grad), rows(self.next_grad), K.ResidualGrad(self.shape, **g),
                                  K.workspace(ctx.residual_workspace_bytes(self.shape)))
        return g

    def wanted_grad(self):
        clean = lambda t: None if t is None else np.nan_to_num(self.made.host(t))  # noqa: E731
        return self.want.grad(clean(self.sum_grad), clean(self.next_grad))


RES = (8192 ** 0.5 / 2 + 20) * U


@pytest.mark.parametrize("c", RESIDUAL, ids=label)
def test_norms_gate_and_sum(env, c):
    call = ResidualCall(env, c)
    total, after = call.forward()
    close(total, call.want.sum, "sum", RES)
    if after is not None:
        close(after, call.want.next, "next", RES)


@pytest.mark.parametrize("c", RESIDUAL, ids=label)
def test_gradients_of_norms_gate_and_sum(env, c):
    call = ResidualCall(env, c, seed=1)
    want, got = call.wanted_grad(), call.backward()
    for k, g in got.items():
        if g is not None:
            close(g, want[k], k, 2 * RES)


def test_gradients_that_are_not_asked_for(env):
    c = residual_case(6, 7, 96, "float32")
    whole = ResidualCall(env, c).backward()
    for leave in (("x",), ("y", "gate"), ("post", "pre"), ("x", "y", "gate"), ("pre", "y")):
        some = ResidualCall(env, c).backward(leave)
        for k, g in some.items():
            assert (g is None) == (k in leave)
            if g is not None:
                assert env[0].equal(g, whole[k]), k


def test_only_one_of_the_two_outputs(env):
    torch, K, ctx = env
    call = ResidualCall(env, residual_case(6, 7, 96, "bfloat16"))
    total, after = call.forward()
    alone, next_alone = call.outs()
    ctx.pql_residual_forward(call.shape, call.given, K.Rows(alone), None)
    ctx.pql_residual_forward(call.shape, call.given, None, K.Rows(next_alone))
    assert torch.equal(alone, total) and torch.equal(next_alone, after)


def test_outputs_in_the_inputs_places(env):
    torch, K, ctx = env
    for c in (residual_case(50, 3, 520, "float32"), residual_case(50, 3, 2048, "bfloat16", groups=16, gate="part")):
        call = ResidualCall(env, c, seed=3)
        total, after = call.forward()
        grads = call.backward()
        x, y = call.x.clone(), call.y.clone()
        given = K.ResidualInput(call.shape, x, y, call.gate, call.post, call.pre, call.lengths)
        ctx.pql_residual_forward(call.shape, given, K.Rows(x), K.Rows(y))
        assert torch.equal(x, total) and torch.equal(y, after)
        dx, dy = call.sum_grad.clone(), call.next_grad.clone()
        ctx.pql_residual_backward(call.shape, call.given, K.Rows(dx), K.Rows(dy), K.ResidualGrad(call.shape, x=dx, y=dy), None)
        assert torch.equal(dx, grads["x"]) and torch.equal(dy, grads["y"])


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("dim,groups", [(64, 1), (96, 3), (2048, 1), (4096, 8)])
def test_rows_that_do_not_count_meet_no_weights(env, dim, groups, dtype):
    """Zeros where nothing counts, and no part in any gradient, also under weights that are not finite."""
    torch, K, ctx = env
    n, t, dt = 5, 7, getattr(torch, dtype)
    odd = lambda: torch.tensor([float("inf"), float("nan"), -float("inf"), 1.0] * (dim // 4), device="cuda")  # noqa: E731
    rows = lambda: torch.full((n, t, dim), float("nan"), dtype=dt, device="cuda")  # noqa: E731
    shape = K.residual_shape(n, t, dim, dt, groups=groups, gate_cols=dim, gate_act="silu", eps_post=1e-5, eps_pre=1e-5)
    given = K.ResidualInput(shape, rows(), rows(), rows(), odd(), odd(), torch.zeros(n, dtype=torch.int32, device="cuda"))
    got = {k: rows() for k in ("sum", "next", "x", "y", "gate")}
    got.update({k: torch.full((dim,), float("nan"), device="cuda") for k in ("post", "pre")})
    ctx.pql_residual_forward(shape, given, K.Rows(got["sum"]), K.Rows(got["next"]))
    grads = K.ResidualGrad(shape, **{k: got[k] for k in ("x", "y", "gate", "post", "pre")})
    work = K.workspace(ctx.residual_workspace_bytes(shape))
    ctx.pql_residual_backward(shape, given, K.Rows(rows()), K.Rows(rows()), grads, work)
    for k, x in got.items():
        assert torch.equal(x, torch.zeros_like(x)), k


def test_rows_that_repeat(env):
    """One row of x for all of them: every repetition has its own gradient."""
    torch, K, ctx = env
    call = ResidualCall(env, residual_case(4, 6, 160, "float32"), seed=4)
    one = call.x[:1, :1]
    spread = K.ResidualInput(call.shape, one.expand(4, 6, 160).contiguous(), call.y, call.gate, call.post, call.pre)
    same = K.ResidualInput(call.shape, one.contiguous().as_strided((4, 6, 160), (0, 0, 1)), call.y, call.gate, call.post, call.pre)
    assert same.c.x.stride == 0
    results = []
    for given in (spread, same):
        total, after = call.outs()
        ctx.pql_residual_forward(call.shape, given, K.Rows(total), K.Rows(after))
        dx = call.outs()[0]
        ctx.pql_residual_backward(call.shape, given, K.Rows(call.sum_grad), K.Rows(call.next_grad), K.ResidualGrad(call.shape, x=dx), None)
        results.append((total, after, dx))
    assert all(torch.equal(a, b) for a, b in zip(*results))


@pytest.mark.parametrize("by", [1e-15, 1e-6, 1e6, 1e15])
def test_sizes_of_values(env, by):
    call = ResidualCall(env, residual_case(4, 6, 160, "float32"), seed=5, by=by)
    total, after = call.forward()
    close(total, call.want.sum, "sum", RES)
    close(after, call.want.next, "next", RES)
    for k, g in call.backward().items():
        close(g, call.wanted_grad()[k], k, 2 * RES)


def test_large_gates(env):
    torch, K, ctx = env
    for act in ("sigmoid", "silu", "gelu", "relu"):
        call = ResidualCall(env, residual_case(2, 2, 64, "float32", act=act), seed=6)
        call.gate.copy_(torch.tensor([-3e38, -1e4, -100.0, -0.0, 0.0, 30.0, 100.0, 60.0], device="cuda").repeat(2, 2, 8))
        h = call.made.host
        with np.errstate(all="ignore"):
            call.want = O.Residual(h(call.x), h(call.y), h(call.gate), h(call.post), h(call.pre), 1, act, *call.eps, *call.scales)
            want = call.wanted_grad()
        close(call.forward()[0], call.want.sum, "sum", RES)
        for k, g in call.backward().items():
            close(g, want[k], k, 2 * RES)


# ---- gated feed-forward block ----------------------------------------------------------------------------------
FFN = [
    # batch, steps, dim, hidden, dtype, act, layout, lengths
    (1, 1, 1, 1, "float32", "silu", "dense", None),
    (1, 1, 8, 8, "bfloat16", "silu", "dense", None),
    (1, 1, 1024, 4096, "bfloat16", "silu", "dense", None),
    (64, 1, 256, 1024, "float32", "gelu", "dense", None),
    (3, 7, 203, 677, "float32", "silu", "offset", [7, 0, 3]),
    (2, 16, 200, 72, "bfloat16", "relu", "wide", [20, -1]),
    (5, 13, 100, 333, "bfloat16", "sigmoid", "offset", None),
    (1, 65, 64, 64, "float32", "silu", "dense", None),
    (1, 65, 64, 64, "bfloat16", "silu", "dense", None),
    (3, 50, 128, 256, "bfloat16", "gelu", "dense", None),
    (3, 50, 128, 256, "float32", "none", "dense", [50, 1, 0]),
    (5, 33, 203, 677, "float32", "silu", "offset", [33, 0, 1, 12, 40]),
    (5, 33, 203, 677, "bfloat16", "gelu", "offset", [33, 0, 1, 12, 40]),
    (7, 40, 72, 136, "bfloat16", "silu", "wide", [0, 40, 39, 0, 0, 7, 40]),
    (130, 1, 9, 5, "float32", "sigmoid", "dense", [1, 0] * 65),
    (6, 64, 520, 1104, "float32", "silu", "wide", None),
    (6, 64, 520, 1104, "bfloat16", "silu", "dense", None),
    (2, 80, 64, 4096, "bfloat16", "silu", "dense", None),       # few tiles, a long contraction
    (2, 80, 1024, 40, "float32", "gelu", "dense", [80, 33]),
    (4, 512, 48, 48, "float32", "silu", "dense", None),         # many rows, small weights
    (700, 3, 16, 24, "bfloat16", "relu", "dense", list(range(-350, 350))),
    (3, 30, 64, 128, "float32", "silu", "dense", [0, 0, 0]),
]


class FfnCall:
    def __init__(self, env, case, seed=0, by=1.0):
        torch, K, ctx = self.env = env
        n, t, d, f, dtype, act, layout, lengths = self.case = case
        self.made = m = Made(env, seed, dtype, layout, lengths)
        self.x, self.out_grad = m.normal(n, t, d, by=by), m.normal(n, t, d)
        self.gate, self.up, self.down = m.normal(f, d, by=d ** -0.5), m.normal(f, d, by=d ** -0.5), m.normal(d, f, by=f ** -0.5)
        m.lengths = None
        self.lengths = lengths_of(torch, lengths)
        self.shape = K.ffn_shape(self.x, self.gate, act)
        self.given = K.FfnInput(self.shape, self.x, self.gate, self.up, self.down, self.lengths)
        h = [np.nan_to_num(m.host(z)) for z in (self.x, self.gate, self.up, self.down)]
        self.want = O.ffn(*h, act, lengths)
        self.want_grad = O.ffn_grad(*h, act, np.nan_to_num(m.host(self.out_grad)), lengths)

    def space(self, call):
        torch, K, ctx = self.env
        s = K.workspace(ctx.ffn_workspace_bytes(self.shape, call))
        s.fill_(255)                                    # NaN wherever it is read before it is written
        return s

    def forward(self, keep):
        torch, K, ctx = self.env
        out = self.made.out(*self.x.shape)
        saved = K.workspace(ctx.ffn_saved_bytes(self.shape)) if keep else None
        if keep:
            saved.fill_(255)
        ctx.pql_ffn_forward(self.shape, self.given, K.Rows(out), saved, self.space(K.FFN_FORWARD))
        return out, saved

    def backward(self, saved, leave=()):
        torch, K, ctx = self.env
        g = {k: None if k in leave else self.made.out(*getattr(self, k).shape) for k in ("x", "gate", "up", "down")}
        ctx.pql_ffn_backward(self.shape, self.given, saved, K.Rows(self.out_grad), K.FfnGrad(self.shape, **g),
                             self.space(K.FFN_BACKWARD if saved is not None else K.FFN_BACKWARD_ALONE))
        return g

    def close(self, got, want, what):
        k = max(self.case[0] * self.case[1], self.case[2], self.case[3])
        bound = 3 * (k ** 0.5 + 10) * U
        if self.case[4] == "float32":
            return close(got, want, what, bound)
        # what lies between two products, rounded to bf16: by 2^-8 / sqrt 3 of its norm at most
        off, want = error_of(got, want)
        bound, norm = bound + 2 * 2.0 ** -8 / 3 ** 0.5, np.linalg.norm(want)
        assert np.linalg.norm(off) <= bound * norm, what
        if norm:
            assert np.max(off / np.maximum(norm / np.sqrt(want.size), np.abs(want))) <= 8 * bound, what


@pytest.mark.parametrize("case", FFN, ids=label)
def test_feed_forward_block(env, case):
    call = FfnCall(env, case)
    out, _ = call.forward(False)
    call.close(out, call.want, "out")
    kept, saved = call.forward(True)
    call.close(kept, call.want, "out with saved")
    again, _ = call.forward(True)
    assert env[0].equal(kept, again)


# Rows around the sizes where other kernels, or other shares of the rows for a workgroup, take over: by the rows, by how many outputs
# there are and by the bytes of the weights.
FEW = [(rows, 1, d, f, dtype, "silu", "dense", None)
       for dtype in ("float32", "bfloat16")
       for rows, d, f in ((32, 24, 3100), (33, 3100, 24), (48, 1600, 1544), (49, 40, 1530), (64, 1530, 40), (65, 64, 3100))]
FEW += [(32, 1, 2048, 4104, "bfloat16", "gelu", "dense", None), (33, 1, 2048, 4104, "bfloat16", "gelu", "dense", None),
        (16, 1, 4096, 8200, "bfloat16", "relu", "dense", None), (17, 1, 4096, 8200, "bfloat16", "relu", "dense", None),
        (40, 1, 2048, 8208, "float32", "silu", "dense", [i % 2 for i in range(40)])]


@pytest.mark.parametrize("case", FEW, ids=label)
def test_feed_forward_block_of_few_rows(env, case):
    call = FfnCall(env, case, seed=4)
    out, _ = call.forward(False)
    call.close(out, call.want, "out")
    assert env[0].equal(out, call.forward(False)[0])


# rounded: by the tiles' kernels once to 8 bits, by those for few rows to 16
@pytest.mark.parametrize("case", [c for c in FFN + FEW if c[4] == "bfloat16" and c[3] * c[0] * c[1] >= 4096], ids=label)
def test_what_lies_between_the_products_is_rounded_once(env, case):
    """Relative to its norm by 2^-9 / sqrt 3 at most (all significands at their smallest; random ones 0.7 of that), or 2^-17 / sqrt 3."""
    call = FfnCall(env, case, seed=10)
    k = max(case[0] * case[1], case[2], case[3])
    bound = 3 * (k ** 0.5 + 10) * U
    few = case[0] * case[1] <= (64 if case[2] * case[3] <= 4 << 20 else 16)
    close(call.forward(False)[0], call.want, "out", bound + 2.0 ** (-17 if few else -9) / 3 ** 0.5)
    out, saved = call.forward(True)
    close(out, call.want, "out with saved", bound + 2.0 ** -9 / 3 ** 0.5)
    for name, g in call.backward(saved).items():
        close(g, call.want_grad[name], name, bound + 2 * 2.0 ** -9 / 3 ** 0.5)


@pytest.mark.parametrize("case", FFN, ids=label)
def test_gradients_of_the_feed_forward_block(env, case):
    call = FfnCall(env, case, seed=1)
    _, saved = call.forward(True)
    first = call.backward(saved)
    for k, g in first.items():
        call.close(g, call.want_grad[k], k)
    for k, g in call.backward(None).items():
        assert env[0].equal(g, first[k]), k + " without saved"


# Enough tiles for the kernels of 256 rows (192 of them), and more than run at a time (256; 512 of 128 x 128 in bf16), so that whole rounds
# go to a workgroup each and the rest is shared out by steps and joined.  By which products: both projections (p), out (o), dm (m), dx (x),
# the weights' gradients (w).
LARGE = [
    (1, 4099, 264, 1032, "float32", "silu", "dense", None),                         # p; 128 rows, whole rounds: m
    (4, 1025, 263, 1029, "float32", "silu", "offset", [1025, 700, 0, 1024]),        # the same by the lengths
    (1, 13400, 520, 520, "float32", "silu", "wide", None),                          # p o m x
    (4, 3350, 517, 520, "float32", "none", "offset", [3350, 0, 3349, 2000]),        # p o m x
    (1, 1000, 1160, 2056, "float32", "silu", "dense", None),                        # w
    (4, 250, 1157, 2051, "float32", "silu", "offset", [250, 3, 249, 0]),            # w
    (1, 13400, 1032, 1032, "bfloat16", "silu", "dense", None),                      # p o m x
    (4, 3350, 1029, 1032, "bfloat16", "silu", "offset", [3350, 0, 3349, 2000]),     # p o m x
    (1, 1000, 2312, 2056, "bfloat16", "silu", "wide", None),                        # w
    (4, 250, 2309, 2051, "bfloat16", "none", "offset", [250, 3, 249, 0]),           # w
    (1, 4099, 1032, 2056, "bfloat16", "silu", "dense", None),                       # p; 128 rows, whole rounds: m
]


@pytest.mark.parametrize("case", LARGE, ids=label)
def test_feed_forward_block_of_many_tiles(env, case):
    """bf16: one rounding of m, da and db, by 2^-9 / sqrt 3 of their norms at most, is passed on as it is by products with terms of random
    signs."""
    call = FfnCall(env, case, seed=9)
    k = max(case[0] * case[1], case[2], case[3])
    bound = 3 * (k ** 0.5 + 10) * U + (2.0 ** -9 / 3 ** 0.5 if case[4] == "bfloat16" else 0.0)
    out, saved = call.forward(True)
    first = call.backward(saved)
    for got, want, what in [(out, call.want, "out")] + [(g, call.want_grad[name], name) for name, g in first.items()]:
        close(got, want, what, bound)
    assert env[0].equal(out, call.forward(False)[0])
    for name, g in call.backward(None).items():
        assert env[0].equal(g, first[name]), name + " without saved"
    if case[7] is not None:
        real = env[0].tensor(O.counted(call.x.shape[:2], case[7]), device="cuda")
        assert not bool(out[~real].any()) and not bool(first["x"][~real].any())


def test_projections_of_different_layouts(env):
    torch, K, ctx = env
    for dtype in ("bfloat16", "float32"):
        call = FfnCall(env, (3, 50, 136, 264, dtype, "silu", "dense", None), seed=3)
        whole = call.forward(False)[0], call.backward(None)
        for wide, at in ((160, 8), (144, 8), (139, 1)):
            for which in ("gate", "up"):
                big = torch.full((264, wide), float("nan"), dtype=call.x.dtype, device="cuda")
                big[:, at:at + 136] = getattr(call, which)
                weights = dict(gate=call.gate, up=call.up, down=call.down)
                weights[which] = big[:, at:at + 136]
                call.given = K.FfnInput(call.shape, call.x, **weights)
                assert torch.equal(call.forward(False)[0], whole[0])
                for k, g in call.backward(None).items():
                    assert torch.equal(g, whole[1][k]), k


@pytest.mark.parametrize("odd", [None, float("inf"), float("nan"), 3.4e38, 1e-39])
@pytest.mark.parametrize("rows,d,f,lengths", [(65, 264, 520, None), (300, 136, 72, [1, 0] * 150), (760, 40, 1048, None), (9, 8, 8, None)])
def test_32_bit_weights_as_they_are_and_as_planes(env, rows, d, f, lengths, odd):
    """Weights whose rows start on 16-byte boundaries and others take two ways to the same terms: equal bits."""
    torch, K, ctx = env
    call = FfnCall(env, (rows, 1, d, f, "float32", "silu", "dense", lengths), seed=6)
    weights = [call.gate, call.up, call.down]
    if odd is not None:
        for w in weights:
            w[w.shape[0] // 2, w.shape[1] // 3] = odd
    def within(w, before, behind):
        wide = torch.full((w.shape[0], before + w.shape[1] + behind), float("nan"), device="cuda")
        wide[:, before:before + w.shape[1]] = w
        return wide[:, before:before + w.shape[1]]

    got = []
    for w in (weights, [within(x, 1, 2) for x in weights], [within(x, 8, 4) for x in weights]):
        call.given = K.FfnInput(call.shape, call.x, *w, call.lengths)
        out, saved = call.forward(True)
        got.append(dict(call.backward(saved), out=out))
    for other in got[1:]:
        for k, x in got[0].items():
            assert torch.equal(x.view(torch.int32), other[k].view(torch.int32)), k
    if odd is None:
        call.close(got[0]["out"], call.want, "out")
        for k, want in call.want_grad.items():
            call.close(got[0][k], want, k)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows", [12, 150])
def test_feed_forward_rows_that_repeat_or_overlap(env, dtype, rows):
    """Tokens, the output's gradient and weights may; results are those of rows of their own."""
    torch, K, ctx = env
    d, f, dt = 40, 72, getattr(torch, dtype)

    def strided(n, cols, stride, by):
        flat = torch.randn((n - 1) * stride + cols, device="cuda").mul_(by).to(dt)
        return flat.as_strided((n, cols), (stride, 1))

    for stride in (0, 8, 37):
        x, grad = (strided(rows, d, stride, 1.0).view(rows, 1, d) if stride else strided(rows, d, 0, 1.0)[:, None] for _ in range(2))
        weights = [strided(f, d, stride, d ** -0.5), strided(f, d, stride, d ** -0.5), strided(d, f, stride, f ** -0.5)]
        shape = K.ffn_shape(x, weights[0], "silu")
        results = []
        for tensors in ((x, *weights, grad), [t.clone(memory_format=torch.contiguous_format) for t in (x, *weights, grad)]):
            *given, do = tensors
            assert K.Rows(given[0]).c.stride == (stride if given[0] is x else d)
            out = torch.empty(rows, 1, d, dtype=dt, device="cuda")
            grads = [torch.empty(t.shape, dtype=dt, device="cuda") for t in given]
            ctx.pql_ffn_forward(shape, K.FfnInput(shape, *given), K.Rows(out), None, K.workspace(ctx.ffn_workspace_bytes(shape, K.FFN_FORWARD)))
            ctx.pql_ffn_backward(shape, K.FfnInput(shape, *given), None, K.Rows(do), K.FfnGrad(shape, *grads),
                                 K.workspace(ctx.ffn_workspace_bytes(shape, K.FFN_BACKWARD_ALONE)))
            results.append((out, *grads))
        assert all(torch.equal(a, b) for a, b in zip(*results))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows", [3, 70])
@pytest.mark.parametrize("d,f", [(65536, 16), (24, 65536), (65535, 9)])
def test_the_widest_feed_forward_blocks(env, dtype, rows, d, f):
    call = FfnCall(env, (rows, 1, d, f, dtype, "silu", "dense", None), seed=11)
    out, saved = call.forward(True)
    call.close(call.forward(False)[0], call.want, "out")
    call.close(out, call.want, "out with saved")
    for k, g in call.backward(saved).items():
        call.close(g, call.want_grad[k], k)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_weights_whose_rows_are_far_apart(env, dtype):
    """At the largest stride of weights that are read where they are, and beyond it."""
    torch, K, ctx = env
    call = FfnCall(env, (150, 1, 40, 264, dtype, "silu", "dense", None), seed=12)
    want = call.forward(False)[0], call.backward(None)
    for stride in (1 << 20, (1 << 20) + 8):
        big = torch.empty(3 * 264 * stride, dtype=call.x.dtype, device="cuda")
        weights = []
        for i, w in enumerate((call.gate, call.up, call.down)):
            weights.append(big[i * 264 * stride:].as_strided(w.shape, (stride, 1)))
            weights[-1].copy_(w)
        call.given = K.FfnInput(call.shape, call.x, *weights)
        assert torch.equal(call.forward(False)[0], want[0])
        for k, g in call.backward(None).items():
            assert torch.equal(g, want[1][k]), k


def test_feed_forward_gradients_that_are_not_asked_for(env):
    call = FfnCall(env, (3, 50, 136, 260, "float32", "silu", "dense", [50, 20, 0]), seed=2)
    _, saved = call.forward(True)
    whole = call.backward(saved)
    for leave in (("x",), ("gate",), ("down", "up"), ("x", "gate", "up", "down"), ("gate", "up", "down")):
        for k, g in call.backward(saved, leave).items():
            assert (g is None) == (k in leave)
            assert g is None or env[0].equal(g, whole[k]), k


# ---- calls as programs make them ---------------------------------------------------------------------------------
def every_call(env, dtype="bfloat16", lengths=(40, 7, 0, 33), seed=7):
    """One of each call on inputs of its own, as (run, inputs, outputs): run(stream) writes the outputs from the inputs."""
    torch, K, ctx = env
    lengths = None if lengths is None else list(lengths)
    made, tokens, _, table, out_grad, lens = embed_inputs(env, (4, 40, 3, 90, 136, dtype, "dense", lengths, "any"), seed)
    shape = K.embed_shape(tokens, table, 0.5)
    out, dtable, space = torch.empty_like(out_grad), torch.empty_like(table), K.workspace(ctx.embed_workspace_bytes(shape))

    def embed(stream=None):
        ctx.pql_embed_forward(shape, tokens, lens, K.Rows(table), K.Rows(out), stream)
        ctx.pql_embed_backward(shape, tokens, lens, K.Rows(out_grad), K.Rows(dtable), space, stream)
    yield embed, [table, out_grad], [out, dtable]

    r = ResidualCall(env, residual_case(4, 40, 136, dtype, groups=2, lengths=lengths), seed)
    total, after = r.outs()
    grads = {k: torch.empty_like(getattr(r, k)) for k in ("x", "y", "gate", "post", "pre")}
    rgrad, rspace = K.ResidualGrad(r.shape, **grads), K.workspace(ctx.residual_workspace_bytes(r.shape))

    def residual(stream=None):
        ctx.pql_residual_forward(r.shape, r.given, K.Rows(total), K.Rows(after), stream)
        ctx.pql_residual_backward(r.shape, r.given, K.Rows(r.sum_grad), K.Rows(r.next_grad), rgrad, rspace, stream)
    yield residual, [r.x, r.y, r.gate], [total, after, *grads.values()]

    f = FfnCall(env, (4, 40, 136, 264, dtype, "silu", "dense", lengths), seed)
    result, fgrads = torch.empty_like(f.x), {k: torch.empty_like(getattr(f, k)) for k in ("x", "gate", "up", "down")}
    fgrad, saved = K.FfnGrad(f.shape, **fgrads), K.workspace(ctx.ffn_saved_bytes(f.shape))
    fspace = K.workspace(max(ctx.ffn_workspace_bytes(f.shape, c) for c in (K.FFN_FORWARD, K.FFN_BACKWARD)))

    def ffn(stream=None):
        ctx.pql_ffn_forward(f.shape, f.given, K.Rows(result), saved, fspace, stream)
        ctx.pql_ffn_backward(f.shape, f.given, saved, K.Rows(f.out_grad), fgrad, fspace, stream)
    yield ffn, [f.x, f.gate, f.out_grad], [result, *fgrads.values()]

    few = FfnCall(env, (10, 1, 136, 264, dtype, "silu", "dense", None), seed)
    one, space1 = torch.empty_like(few.x), K.workspace(ctx.ffn_workspace_bytes(few.shape, K.FFN_FORWARD))
    yield (lambda stream=None: ctx.pql_ffn_forward(few.shape, few.given, K.Rows(one), None, space1, stream)), [few.x, few.gate], [one]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_calls_repeat_bit_for_bit_on_another_stream_and_in_graphs(env, dtype):
    torch = env[0]
    for run, inputs, outputs in every_call(env, dtype):
        run()
        first = [x.clone() for x in outputs]
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        for x in outputs:
            x.fill_(7)
        stream.wait_stream(torch.cuda.current_stream())
        run(stream)
        stream.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, outputs))
        # two graphs that share the call's workspace, replayed in turn, with eager work and other inputs between
        graphs = []
        for _ in range(2):
            graphs.append(torch.cuda.CUDAGraph())
            with torch.cuda.graph(graphs[-1]):
                run()
        for i in range(4):
            for x in inputs:
                x.mul_(1.25)
            run()
            want = [x.clone() for x in outputs]
            for x in outputs:
                x.zero_()
            graphs[i % 2].replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(want, outputs)), i


def test_calls_of_two_contexts_at_once(env):
    """Two streams, contexts and workspaces: the calls of one do not meet those of the other."""
    torch, K, _ = env
    sets = [list(every_call((torch, K, K.BlockContext()), "float32", seed=s)) for s in (1, 2)]
    for calls in sets:
        for run, _, _ in calls:
            run()
    torch.cuda.synchronize()
    want = [[[x.clone() for x in outputs] for _, _, outputs in calls] for calls in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    for calls in sets:
        for _, _, outputs in calls:
            for x in outputs:
                x.zero_()
    torch.cuda.synchronize()
    for _ in range(5):
        for i in range(len(sets[0])):
            for calls, stream in zip(sets, streams):
                calls[i][0](stream)
    torch.cuda.synchronize()
    for calls, kept in zip(sets, want):
        for (_, _, outputs), w in zip(calls, kept):
            assert all(torch.equal(a, b) for a, b in zip(w, outputs))


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan"), 3.0e38])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_values_that_are_not_finite_stay_in_their_row(env, dtype, bad):
    """Of tokens' results; the weights' gradients are sums over all rows."""
    torch, K, ctx = env
    for rows in ((4, 40), (10, 1)):
        f, clean = (FfnCall(env, (*rows, 136, 264, dtype, "silu", "dense", None), 5) for _ in range(2))
        f.x[1, 0, 3] = bad
        keep = torch.ones(rows, dtype=torch.bool, device="cuda")
        keep[1, 0] = False
        for save in (False, True):
            (a, sa), (b, sb) = f.forward(save), clean.forward(save)
            assert torch.equal(a[keep], b[keep])
        assert torch.equal(f.backward(sa)["x"][keep], clean.backward(sb)["x"][keep])
    r, clean = (ResidualCall(env, residual_case(4, 40, 136, dtype, groups=2), 5) for _ in range(2))
    r.y[1, 0, 3] = bad
    keep = torch.ones(4, 40, dtype=torch.bool, device="cuda")
    keep[1, 0] = False
    assert all(torch.equal(a[keep], b[keep]) for a, b in zip(r.forward(), clean.forward()))
    got, want = r.backward(), clean.backward()
    assert all(torch.equal(got[k][keep], want[k][keep]) for k in ("x", "y", "gate"))


def test_values_of_any_size_in_three_terms(env):
    """fp32 values of very different sizes: each product is as exact as in fp32, relative to the sum of the terms' sizes."""
    torch, K, ctx = env
    rng = np.random.default_rng(3)
    d, f = 128, 64
    spread = lambda *s: rng.standard_normal(s) * 10.0 ** rng.uniform(-12, 12, s)  # noqa: E731
    dev = lambda x: torch.tensor(x).float().cuda()  # noqa: E731
    x, gate, up, down = dev(spread(1, 100, d)), dev(1e-14 * rng.standard_normal((f, d))), dev(spread(f, d)), dev(spread(d, f))
    shape = K.ffn_shape(x, gate, "none")
    out = torch.empty_like(x)
    ctx.pql_ffn_forward(shape, K.FfnInput(shape, x, gate, up, down), K.Rows(out), K.workspace(ctx.ffn_saved_bytes(shape)),
                        K.workspace(ctx.ffn_workspace_bytes(shape, K.FFN_FORWARD)))
    h = [t.double().cpu().numpy() for t in (x, gate, up, down)]
    size = (np.abs(h[0]) @ np.abs(h[1]).T * (np.abs(h[0]) @ np.abs(h[2]).T)) @ np.abs(h[3]).T
    # three products of at most 128 terms, each off by 128 roundings and the three left out terms
    assert np.all(np.abs(out.double().cpu().numpy() - O.ffn(*h, "none")) <= 3 * (128 + 4) * U * size)


def test_places_further_apart_than_32_bits_reach(env):
    torch, K, ctx = env
    # a table of 2^31 elements and more
    vocab, dim = 70000, 32768
    table = torch.empty(vocab, dim, dtype=torch.bfloat16, device="cuda")
    at = torch.tensor([[0], [vocab - 1], [35000], [vocab - 1]], dtype=torch.int32, device="cuda").view(1, 4, 1)
    table[0], table[vocab - 1], table[35000] = 1, 2, 3
    out = torch.empty(1, 4, dim, dtype=torch.bfloat16, device="cuda")
    shape = K.embed_shape(at, table, 0.5)
    ctx.pql_embed_forward(shape, at, None, K.Rows(table), K.Rows(out))
    assert [float(out[0, i].min()) for i in range(4)] == [0.5, 1.0, 1.5, 1.0] == [float(out[0, i].max()) for i in range(4)]
    ctx.pql_embed_backward(shape, at, None, K.Rows(out), K.Rows(table), K.workspace(ctx.embed_workspace_bytes(shape)))
    rows = table.float().sum(1)
    want = torch.zeros_like(rows)
    want[0], want[vocab - 1], want[35000] = 0.25 * dim, dim, 0.75 * dim
    assert torch.equal(rows, want)
    del table
    # rows 2^20 elements apart, 2100 of them
    big = torch.empty(2100 * (1 << 20), dtype=torch.bfloat16, device="cuda")
    far = big.as_strided((2100, 1, 64), (1 << 20, 1 << 20, 1))
    near = torch.randn(2100, 1, 64, device="cuda").bfloat16()
    far.copy_(near)
    weights = [torch.randn(*s, device="cuda").mul_(0.1).bfloat16() for s in ((64, 64), (64, 64), (64, 64))]
    shape = K.ffn_shape(near, weights[0], "silu")
    given = [K.FfnInput(shape, x, *weights) for x in (near, far)]
    outs = [torch.empty_like(near) for _ in range(2)]
    grads = [[torch.empty_like(t) for t in (near, *weights)] for _ in range(2)]
    do = torch.randn_like(near)
    for g, o, dg in zip(given, outs, grads):
        ctx.pql_ffn_forward(shape, g, K.Rows(o), None, K.workspace(ctx.ffn_workspace_bytes(shape, K.FFN_FORWARD)))
        ctx.pql_ffn_backward(shape, g, None, K.Rows(do), K.FfnGrad(shape, *dg), K.workspace(ctx.ffn_workspace_bytes(shape, K.FFN_BACKWARD_ALONE)))
    assert torch.equal(*outs) and all(torch.equal(a, b) for a, b in zip(*grads))
    shape = K.residual_shape(2100, 1, 64, torch.bfloat16, eps_pre=1e-5)
    results = [torch.empty_like(near) for _ in range(2)]
    for x, o in zip((near, far), results):
        ctx.pql_residual_forward(shape, K.ResidualInput(shape, x), None, K.Rows(o))
    assert torch.equal(*results)
    ctx.pql_residual_forward(shape, K.ResidualInput(shape, near), None, K.Rows(far))
    assert torch.equal(far, results[0])


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_rows_calls_leave_what_is_not_theirs(env, dtype):
    """Neither the gaps between rows nor what lies behind the last one are written, by results or gradients."""
    torch, K, ctx = env
    dt = getattr(torch, dtype)

    def framed(n, cols):
        big = torch.full((n + 3, cols + 16), 7.0, dtype=dt, device="cuda")
        return big, big[:n, 8:8 + cols]

    for cols, hidden in ((136, 264), (61, 35)):
        for rows in (12, 150):                          # few rows, tiles
            x, do = (torch.randn(rows, 1, cols, device="cuda").to(dt) for _ in range(2))
            weights = [torch.randn(*s, device="cuda").mul_(0.1).to(dt) for s in ((hidden, cols), (hidden, cols), (cols, hidden))]
            shape = K.ffn_shape(x, weights[0], "silu")
            given = K.FfnInput(shape, x, *weights)
            out, grads = framed(rows, cols), [framed(rows, cols), framed(hidden, cols), framed(hidden, cols), framed(cols, hidden)]
            ctx.pql_ffn_forward(shape, given, K.Rows(out[1]), None, K.workspace(ctx.ffn_workspace_bytes(shape, K.FFN_FORWARD)))
            ctx.pql_ffn_backward(shape, given, None, K.Rows(do), K.FfnGrad(shape, *[g[1] for g in grads]),
                                 K.workspace(ctx.ffn_workspace_bytes(shape, K.FFN_BACKWARD_ALONE)))
            shape = K.residual_shape(rows, 1, cols, dt, gate_cols=cols, gate_act="silu", eps_post=1e-5, eps_pre=1e-5)
            given = K.ResidualInput(shape, x, do, x)
            more = [framed(rows, cols) for _ in range(5)]
            ctx.pql_residual_forward(shape, given, K.Rows(more[0][1]), K.Rows(more[1][1]))
            ctx.pql_residual_backward(shape, given, K.Rows(do), K.Rows(x), K.ResidualGrad(shape, *[m[1] for m in more[2:]]), None)
            for big, inner in [out] + grads + more:
                n, c = inner.shape
                assert bool((big[n:] == 7).all()) and bool((big[:, :8] == 7).all()) and bool((big[:, 8 + c:] == 7).all())
                assert not bool((inner == 7).all(1).any())


def test_no_rows_at_all(env):
    """Gradients of weights are written all the same."""
    torch, K, ctx = env
    x, tokens = torch.empty(0, 5, 24, device="cuda"), torch.empty(0, 5, 2, dtype=torch.int32, device="cuda")
    weights = [torch.randn(*s, device="cuda") for s in ((40, 24), (40, 24), (24, 40))]
    shape = K.ffn_shape(x, weights[0], "silu")
    given, grads = K.FfnInput(shape, x, *weights), [torch.full_like(w, 7) for w in weights]
    ctx.pql_ffn_backward(shape, given, None, K.Rows(x), K.FfnGrad(shape, None, *grads), None)
    table, dtable = torch.randn(9, 24, device="cuda"), torch.full((9, 24), 7.0, device="cuda")
    shape = K.embed_shape(tokens, table, 1.0)
    ctx.pql_embed_backward(shape, tokens, None, K.Rows(x), K.Rows(dtable), None)
    shape = K.residual_shape(0, 5, 24, torch.float32, eps_post=1e-5, eps_pre=1e-5)
    post, pre = torch.full((24,), 7.0, device="cuda"), torch.full((24,), 7.0, device="cuda")
    ctx.pql_residual_backward(shape, K.ResidualInput(shape, x, x), K.Rows(x), K.Rows(x), K.ResidualGrad(shape, post=post, pre=pre), None)
    assert all(not bool(t.any()) for t in grads + [dtable, post, pre])


def test_lengths_that_change_between_replays(env):
    torch = env[0]
    for run, _, outputs in every_call(env, "float32"):
        calls = [c.cell_contents for c in run.__closure__ if c.cell_contents is not None]
        lengths = next((c for c in calls if isinstance(c, torch.Tensor) and c.dtype is torch.int32 and c.shape == (4,)), None)
        if lengths is None:
            lengths = next((getattr(c, "lengths", None) for c in calls if getattr(c, "lengths", None) is not None), None)
        if lengths is None:
            continue
        graph = torch.cuda.CUDAGraph()
        run()
        with torch.cuda.graph(graph):
            run()
        for new in ([33, 0, 7, 33], [0, 0, 0, 0], [33, 7, 0, 33], [1, 7, 0, 0]):       # within what is not poisoned, or nothing that is
            lengths.copy_(torch.tensor([min(a, b) for a, b in zip(new, (40, 7, 0, 33))], dtype=torch.int32))
            run()
            want = [x.clone() for x in outputs]
            for x in outputs:
                x.fill_(7)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(want, outputs)), new


def test_more_rows_than_a_grid_holds_workgroups_for(env):
    torch, K, ctx = env
    rows, dim = (1 << 24) + 5, 1032
    table = torch.randn(11, dim, device="cuda").bfloat16()
    tokens = torch.arange(rows, dtype=torch.int32, device="cuda").remainder_(11).view(1, rows, 1)
    out = torch.empty(1, rows, dim, dtype=torch.bfloat16, device="cuda")
    shape = K.embed_shape(tokens, table, 1.0)
    ctx.pql_embed_forward(shape, tokens, None, K.Rows(table), K.Rows(out))
    for at in (0, 1 << 22, 1 << 23, rows - 11):
        assert torch.equal(out[0, at:at + 11], table[tokens[0, at:at + 11, 0].long()])


def test_as_many_rows_as_a_feed_forward_call_takes(env):
    """2^22 tiles of one column; small whole numbers, so that results are exact."""
    torch, K, ctx = env
    rows = (1 << 30) - 1
    x = torch.randint(-3, 4, (1, rows, 1), dtype=torch.int8, device="cuda").bfloat16()
    one = torch.ones(1, 1, dtype=torch.bfloat16, device="cuda")
    shape = K.ffn_shape(x, one, "none")
    out = torch.empty_like(x)
    ctx.pql_ffn_forward(shape, K.FfnInput(shape, x, one, one, one), K.Rows(out), None, K.workspace(ctx.ffn_workspace_bytes(shape, K.FFN_FORWARD)))
    assert torch.equal(out, x * x)


@pytest.mark.parametrize("dtype,rows", [("bfloat16", (1 << 28) + 77), ("float32", (1 << 26) + 77)])
def test_gradients_of_sums_over_very_many_rows(env, dtype, rows):
    """Of which a few, far apart, are not zero; small whole numbers, so that results are exact."""
    torch, K, ctx = env
    dt = getattr(torch, dtype)
    at = torch.tensor([0, 63, 64, 4095, rows // 3, rows // 2, rows - 78, rows - 1], device="cuda")
    x, grad = (torch.zeros(1, rows, 8, dtype=dt, device="cuda") for _ in range(2))
    few = torch.randint(-2, 3, (2, len(at), 8), device="cuda")
    x[0, at], grad[0, at] = few[0].to(dt), few[1].to(dt)
    weights = [torch.randint(-1, 2, (8, 8), device="cuda").to(dt) for _ in range(3)]
    shape = K.ffn_shape(x, weights[0], "none")
    got = [torch.empty_like(t) for t in (x, *weights)]
    ctx.pql_ffn_backward(shape, K.FfnInput(shape, x, *weights), None, K.Rows(grad), K.FfnGrad(shape, *got),
                         K.workspace(ctx.ffn_workspace_bytes(shape, K.FFN_BACKWARD_ALONE)))
    h = [t.double().cpu().numpy() for t in (few[0].view(1, -1, 8), *weights)]
    want = O.ffn_grad(*h, "none", few[1].view(1, -1, 8).double().cpu().numpy())
    exact = lambda g, w: np.array_equal(g.double().cpu().numpy(), torch.tensor(w).to(dt).double().numpy())  # noqa: E731
    assert exact(got[0][0, at], want["x"][0]) and int(got[0].count_nonzero()) == np.count_nonzero(want["x"])
    assert all(exact(g, want[k]) for g, k in zip(got[1:], ("gate", "up", "down")))


def test_the_widest_embeddings(env):
    """2^24 columns on no 16-byte boundary, in runs that cross the ends of two chunks."""
    torch, K, ctx = env
    dim, n = 1 << 24, 37
    grad = torch.randint(-8, 9, (1, n, dim + 1), dtype=torch.int8, device="cuda").bfloat16()[..., 1:]
    tokens = torch.zeros(1, n, 1, dtype=torch.int32, device="cuda")
    tokens[0, -1] = 1
    table = torch.empty(2, dim + 1, dtype=torch.bfloat16, device="cuda")[:, 1:]
    shape = K.embed_shape(tokens, table, 0.25)
    ctx.pql_embed_backward(shape, tokens, None, K.Rows(grad), K.Rows(table), K.workspace(ctx.embed_workspace_bytes(shape)))
    want = sum(grad[0, i].float() for i in range(n - 1)) * 0.25
    assert torch.equal(table[0], want.bfloat16()) and torch.equal(table[1], grad[0, -1] * 0.25)
    out = torch.empty_like(grad)
    ctx.pql_embed_forward(shape, tokens, None, K.Rows(table), K.Rows(out))
    assert torch.equal(out[0, 0], (table[0].float() * 0.25).bfloat16()) and torch.equal(out[0, -1], table[1] * 0.25)


@pytest.mark.parametrize("vocab", [3, 700, 40000])
@pytest.mark.parametrize("which", ["equal", "in turn", "runs", "pairs", "any"])
def test_every_place_is_counted_once(env, vocab, which):
    """More places than are sorted in one launch, in patterns that meet in one wavefront; whole numbers, whose sums are exact."""
    torch, K, ctx = env
    n, dim = 20011, 8
    at = torch.arange(n, device="cuda")
    tokens = {"equal": at * 0 + vocab - 1, "in turn": at % min(vocab, 65), "runs": at // 63 % vocab, "pairs": at // 2 * 31 % vocab,
              "any": torch.randint(0, vocab, (n,), device="cuda")}[which].int().view(1, n, 1)
    grad = torch.randint(-8, 9, (1, n, dim), device="cuda").float()
    table = torch.empty(vocab, dim, device="cuda")
    shape = K.embed_shape(tokens, table, 1.0)
    ctx.pql_embed_backward(shape, tokens, None, K.Rows(grad), K.Rows(table), K.workspace(ctx.embed_workspace_bytes(shape)))
    want = np.zeros((vocab, dim))
    np.add.at(want, tokens.flatten().cpu().numpy(), grad[0].double().cpu().numpy())
    assert np.array_equal(table.double().cpu().numpy(), want)


# ---- infinite values -----------------------------------------------------------------------------------------------
def infinite_rows(env, dtype, rows, d, f, lengths=None, act="none", seed=8):
    """A call whose weights' signs and sizes make every result of the rows with an infinite element infinite, of one sign a column."""
    torch, K, ctx = env
    call = FfnCall(env, (1, rows, d, f, dtype, act, "dense", lengths), seed)
    m = call.made
    sign = np.where(np.arange(d) % 3 == 0, -1.0, 1.0)
    size = lambda *s: np.where(m.rng.random(s) < 0.5, 1.0, 1.1 + m.rng.random(s))  # noqa: E731  of one term and of three
    call.gate, call.up = m.place(size(f, d)), m.place(size(f, d))
    call.down = m.place(sign[:, None] * size(d, f))
    at = [r for r in (3, rows // 2) if lengths is None or r < lengths[0]]
    for r in at:
        call.x[0, r], call.out_grad[0, r] = m.place(size(d)), m.place(sign * size(d))
        call.x[0, r, r % d] = float("inf")
    call.given = K.FfnInput(call.shape, call.x, call.gate, call.up, call.down, call.lengths)
    h = [np.nan_to_num(m.host(z), nan=0.0, posinf=np.inf) for z in (call.x, call.gate, call.up, call.down)]
    with np.errstate(invalid="ignore"):
        call.want = O.ffn(*h, act, lengths)
        call.want_grad = O.ffn_grad(*h, act, np.nan_to_num(m.host(call.out_grad)), lengths)
    return call, at


def same_kind(call, got, want, what):
    """Infinite where the definition is, with its sign, NaN where it is, and close to it elsewhere."""
    off = got.double().cpu().numpy()
    finite = np.isfinite(want)
    assert np.array_equal(np.where(finite, 0.0, want), np.where(finite, 0.0, off), equal_nan=True), what
    call.close(got.masked_fill(~call.made.torch.tensor(finite, device="cuda"), 0), np.where(finite, want, 0.0), what)


@pytest.mark.parametrize("rows,d,f", [(9, 13, 21), (70, 13, 21), (70, 24, 37), (300, 61, 203)])
def test_infinite_tokens_next_to_columns_that_are_not_there(env, rows, d, f):
    """Widths of no whole granule in bf16: what stands behind the last column of m and its gradient meets zeros."""
    call, at = infinite_rows(env, "bfloat16", rows, d, f)
    assert all(np.all(np.isinf(call.want[0, r])) and np.all(np.isinf(call.want_grad["x"][0, r])) for r in at)
    outs = call.forward(False)[0], *call.forward(True)
    for out in outs[:2]:
        same_kind(call, out, call.want, "out")
    for saved in (outs[2], None):
        for k, g in call.backward(saved).items():
            same_kind(call, g, call.want_grad[k], k)


# ---- activations far from zero -------------------------------------------------------------------------------------
def gate_values(env, dtype, act, x):
    """act(x) and act'(x) as a residual call and its gradient give them: y and the sum's gradient are ones, there are no norms."""
    torch, K, ctx = env
    gate = torch.tensor(x).to(getattr(torch, dtype)).cuda().view(1, 1, -1)
    one, d = torch.ones_like(gate), gate.shape[-1]
    shape = K.residual_shape(1, 1, d, gate.dtype, gate_cols=d, gate_act=act)
    given = K.ResidualInput(shape, None, one, gate)
    f, slope = torch.empty_like(one), torch.empty_like(one)
    ctx.pql_residual_forward(shape, given, K.Rows(f), None)
    ctx.pql_residual_backward(shape, given, K.Rows(one), None, K.ResidualGrad(shape, gate=slope), None)
    return f, slope, gate.double().cpu().numpy()


@pytest.mark.parametrize("act", ["sigmoid", "silu"])
def test_activations_far_from_zero(env, act):
    """Relative to the terms they are sums of: e = exp(-|x|) is off by 3 u, 1 / (1 + e) by 1.5 + 1 + 2 u, e times that by 7 u at most,
    and the products and sums that follow by u each: 8 u for x s, 14.5 u for either slope."""
    f, slope, x = gate_values(env, "float32", act, np.linspace(-80, 80, 8192))
    s, q = 1 / (1 + np.exp(-x)), 1 / (1 + np.exp(x))
    want, terms = (s, s * q) if act == "sigmoid" else (x * s, s * (1 + np.abs(x) * q))
    assert np.all(np.abs(f.double().cpu().numpy() - want) <= 10 * U * np.abs(want))
    assert np.all(np.abs(slope.double().cpu().numpy() - (s * q if act == "sigmoid" else s * (1 + x * q))) <= 16 * U * terms)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_gelu_far_from_zero(env, dtype):
    """Relative to the terms, beyond the rounding to the type: 7.5 u for the share's polynomial, 3 u for its argument, 2 u for an
    exponential and 3 u for products, and 2.5 u x^2 for the rounding of its exponent; erfc of the library is within 16 u."""
    f, slope, x = gate_values(env, dtype, "gelu", np.linspace(-12, 12, 8192))
    below = 0.5 * np.array([math.erfc(-v / math.sqrt(2)) for v in x.ravel()]).reshape(x.shape)
    far = x * np.exp(-0.5 * x * x) / math.sqrt(2 * math.pi)
    bound = (16 + 2.5 * x * x) * U
    assert np.all(error_of(f, x * below)[0] <= bound * np.abs(x) * below)
    assert np.all(error_of(slope, below + far)[0] <= bound * (below + np.abs(far)))


@pytest.mark.parametrize("act", ["none", "sigmoid"])
@pytest.mark.parametrize("rows,d,f,lengths", [
    (9, 24, 40, None), (64, 264, 520, None), (65, 264, 520, None), (65, 13, 21, None),       # few rows and tiles, aligned weights and others
    (300, 136, 264, [190]), (70, 24, 1544, None), (2100, 40, 24, None)])                      # rows that do not count, joined parts
def test_infinite_tokens_in_32_bits(env, rows, d, f, lengths, act):
    """What fp32 arithmetic gives, whatever the number of rows: three terms of a value must not make NaN of an infinite one."""
    call, at = infinite_rows(env, "float32", rows, d, f, lengths, act)
    assert all(np.all(np.isinf(call.want[0, r])) for r in at)
    outs = call.forward(False)[0], *call.forward(True)
    for out in outs[:2]:
        same_kind(call, out, call.want, "out")
    for saved in (outs[2], None):
        for k, g in call.backward(saved).items():
            same_kind(call, g, call.want_grad[k], k)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows,d,f,lengths", [(4099, 264, 1029, None), (13400, 520, 520, [13300]), (13400, 1032, 1029, None), (1000, 2309, 2056, None)])
def test_infinite_tokens_in_many_tiles(env, rows, d, f, lengths, dtype):
    call, at = infinite_rows(env, dtype, rows, d, f, lengths)
    out, saved = call.forward(True)
    same_kind(call, out, call.want, "out")
    for k, g in call.backward(saved).items():
        same_kind(call, g, call.want_grad[k], k)


@pytest.mark.parametrize("rows", [33, 200])
@pytest.mark.parametrize("which", ["gate", "up", "down"])
@pytest.mark.parametrize("odd", [float("inf"), float("-inf"), float("nan")])
def test_infinite_weights_in_32_bits(env, rows, which, odd, monkeypatch):
    """The activation and its derivative are those of 32 bits: rows of ones sum to a = 120, where the sigmoid's derivative, e^-120 = 8e-53,
    is below half the smallest 32-bit number, 2^-150 = 7e-46, so that it is 0 and an infinite up makes NaN of its product with it."""
    call, _ = infinite_rows(env, "float32", rows, 72, 104, act="sigmoid")
    call.x.copy_(env[0].where(call.x.isinf(), 1.0, call.x))
    getattr(call, which)[5, 7] = odd
    h = [call.made.host(z) for z in (call.x, call.gate, call.up, call.down)]
    exact = O.activate
    monkeypatch.setattr(O, "activate", lambda act, x: tuple(v.astype(np.float32).astype(np.float64) for v in exact(act, x)))
    with np.errstate(invalid="ignore"):
        call.want, call.want_grad = O.ffn(*h, "sigmoid"), O.ffn_grad(*h, "sigmoid", call.made.host(call.out_grad))
    out, saved = call.forward(True)
    same_kind(call, call.forward(False)[0], call.want, "out")
    same_kind(call, out, call.want, "out with saved")
    for k, g in call.backward(saved).items():
        same_kind(call, g, call.want_grad[k], k)


@pytest.mark.parametrize("rows", [12, 33, 200])
@pytest.mark.parametrize("which", ["gate", "up", "down"])
@pytest.mark.parametrize("odd", [float("inf"), float("-inf"), float("nan")])
def test_infinite_weights_in_16_bits(env, rows, which, odd):
    """In calls of few rows as well, whose m has two terms."""
    call, _ = infinite_rows(env, "bfloat16", rows, 72, 104)
    call.x.copy_(env[0].where(call.x.isinf(), 1.0, call.x))
    getattr(call, which)[5, 7] = odd
    h = [call.made.host(z) for z in (call.x, call.gate, call.up, call.down)]
    with np.errstate(invalid="ignore"):
        call.want, call.want_grad = O.ffn(*h, "none"), O.ffn_grad(*h, "none", call.made.host(call.out_grad))
    out, saved = call.forward(True)
    same_kind(call, call.forward(False)[0], call.want, "out")
    same_kind(call, out, call.want, "out with saved")
    for k, g in call.backward(saved).items():
        same_kind(call, g, call.want_grad[k], k)


def test_sums_that_overflow_in_32_bits(env):
    """Products of finite values beyond the largest one: infinite in a call of few rows and in one of many."""
    torch, K, ctx = env
    for rows in (20, 100):
        x = torch.randn(1, rows, 40, device="cuda")
        gate, up, down = (torch.rand(*s, device="cuda") + 0.1 for s in ((56, 40), (56, 40), (40, 56)))
        x[0, 3], x[0, 5] = 3.1e30, -2.7e30                      # m: 1e31 squared
        shape = K.ffn_shape(x, gate, "none")
        out, saved = torch.empty_like(x), K.workspace(ctx.ffn_saved_bytes(shape))
        for keep in (None, saved):
            ctx.pql_ffn_forward(shape, K.FfnInput(shape, x, gate, up, down), K.Rows(out), keep, K.workspace(ctx.ffn_workspace_bytes(shape, K.FFN_FORWARD)))
            odd = out.isinf()
            assert bool((out[0, 3] == float("inf")).all()) and bool((out[0, 5] == float("inf")).all())
            assert int(odd.sum()) == 80 and not bool(out.isnan().any())
