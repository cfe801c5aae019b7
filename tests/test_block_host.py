"""The operators around a student's memory on the host: header, binding, refusals before any launch, and the
double-precision reference's gradients against differences."""
import ctypes as C
import os
import re
import shutil
import subprocess

import numpy as np
import pytest

from oracle import block_oracle as O
from paper_2307_12983_amd import block as K

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "pql_block.h")
P = 0x1000                                      # never dereferenced: validation fails first
INVALID, NULL, ALIGNMENT = -1, -2, -6


def test_library_exports_what_the_header_declares_with_the_bindings_prototypes():
    lib = K.load_library()
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    protos = re.findall(r"\b(int32_t|int64_t)\s+(pql_[a-z_]+)\s*\(([^)]*)\)\s*;", text)
    assert sorted(n for _, n, _ in protos) == sorted(K.EXPORTS)
    scalars = {"int32_t": C.c_int32, "int64_t": C.c_int64, "float": C.c_float}
    for ret, name, params in protos:
        fn = getattr(lib, name)
        assert fn.restype is scalars[ret], name
        plist = [p.strip() for p in params.split(",")]
        assert len(plist) == len(fn.argtypes), name
        for p, t in zip(plist, fn.argtypes):
            assert (t is C.c_void_p or issubclass(t, C._Pointer)) if "*" in p else t is scalars[p.split()[0]], (name, p)


def mirrors():
    names = {"pql_rows": "PqlRows"}
    for op in {e.split("_")[1] for e in K.EXPORTS}:
        for part in ("shape", "input", "grad"):
            cls = "Pql" + op.capitalize() + part.capitalize()
            if hasattr(K, cls):
                names["pql_%s_%s" % (op, part)] = cls
    return {c: getattr(K, p) for c, p in names.items()}


def test_header_is_plain_c_and_the_ctypes_structures_have_its_layout(tmp_path):
    gcc, gxx = shutil.which("gcc"), shutil.which("g++")
    if not gcc or not gxx:
        pytest.skip("no host C compiler")
    for cc, std, lang in ((gcc, "-std=c99", "c"), (gxx, "-std=c++11", "c++")):
        r = subprocess.run([cc, std, "-x", lang, "-Wall", "-Wextra", "-pedantic", "-Werror", "-fsyntax-only", HEADER],
                           capture_output=True, text=True)
        assert r.returncode == 0, r.stderr
    text = open(HEADER).read()
    assert set(re.findall(r"\}\s*(pql_\w+)\s*;", text)) == set(mirrors())
    consts = {m: getattr(K, m) for m in re.findall(r"#define (PQL_\w+_MAX_\w+)", text)}
    consts.update({"PQL_ACT_" + k.upper(): v for k, v in K.ACTIVATIONS.items()})
    consts.update({"PQL_" + k: v for k, v in vars(K).items() if k.startswith("FFN_")})
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "pql_block.h"', "int main(void) {"]
    for cname, cls in mirrors().items():
        lines.append('printf("%s %%zu\\n", sizeof(%s));' % (cname, cname))
        lines += ['printf("%s.%s %%zu\\n", offsetof(%s, %s));' % (cname, f, cname, f) for f, _ in cls._fields_]
    lines += ['printf("%s %%d\\n", %s);' % (n, n) for n in consts] + ["return 0; }"]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines))
    r = subprocess.run([gcc, "-std=c99", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    got = dict(l.split() for l in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.splitlines())
    for cname, cls in mirrors().items():
        assert int(got[cname]) == C.sizeof(cls), cname
        for f, _ in cls._fields_:
            assert int(got["%s.%s" % (cname, f)]) == getattr(cls, f).offset, "%s.%s" % (cname, f)
    for n, x in consts.items():
        assert int(got[n]) == x


def r(x):
    return None if x is None else C.byref(x)


def rows(data=P, stride=64):
    return K.PqlRows(data, stride)


# ---- embeddings ---------------------------------------------------------------------------------------------
def embed_shape(**kw):
    d = dict(batch=2, steps=8, per_row=2, vocab=30, dim=64, dtype=0, scale=1.0)
    d.update(kw)
    return K.PqlEmbedShape(*[d[f] for f, _ in K.PqlEmbedShape._fields_])


def embed_calls(ctx, s, tokens=P, lengths=None, table=rows(), out=rows(), ws=P):
    return (ctx.lib.pql_embed_forward(ctx.h, r(s), tokens, lengths, r(table), r(out), None),
            ctx.lib.pql_embed_backward(ctx.h, r(s), tokens, lengths, r(out), r(table), ws, None))


@pytest.mark.parametrize("kw", [dict(batch=-1), dict(steps=-1), dict(per_row=0), dict(vocab=0), dict(vocab=2 ** 31 - 1), dict(dim=0), dict(dim=1 << 25),
                                dict(dtype=2), dict(scale=float("nan")), dict(scale=float("inf")), dict(batch=1 << 16, steps=1 << 15)])
def test_embeddings_refuse_bad_shapes(kw):
    ctx, s = K.BlockContext(), embed_shape(**kw)
    assert embed_calls(ctx, s) == (INVALID, INVALID) and ctx.embed_workspace_bytes(s) == INVALID
    assert "bad shape" in ctx.last_error()


def test_embeddings_refuse_bad_pointers_and_strides():
    ctx, s = K.BlockContext(), embed_shape()
    both = lambda code, **kw: embed_calls(ctx, s, **kw) == (code, code)  # noqa: E731
    assert embed_calls(ctx, None) == (NULL, NULL) and both(NULL, table=None) and both(NULL, out=None) and both(NULL, tokens=None)
    assert both(NULL, table=rows(None)) and both(NULL, out=rows(None))
    assert both(ALIGNMENT, tokens=P + 2) and both(ALIGNMENT, lengths=P + 2) and both(ALIGNMENT, table=rows(P + 2)) and both(ALIGNMENT, out=rows(P + 1))
    assert both(INVALID, table=rows(stride=-1)) and both(INVALID, out=rows(stride=-64))
    forward, backward = embed_calls(ctx, s, out=rows(stride=0), ws=None)
    assert forward == INVALID and backward == NULL              # an output's rows have places of their own
    assert embed_calls(ctx, s, table=rows(stride=63), ws=P)[1] == INVALID
    assert embed_calls(ctx, s, out=rows(stride=0), ws=P + 16)[1] == ALIGNMENT
    assert ctx.lib.pql_embed_forward(None, r(s), P, None, r(rows()), r(rows()), None) == NULL
    assert ctx.lib.pql_embed_workspace_bytes(None) == NULL


def test_embedding_workspaces():
    ctx = K.BlockContext()
    sizes = [ctx.embed_workspace_bytes(embed_shape(batch=b, vocab=v)) for b in (0, 1, 512, 513, 4096) for v in (1, 1023, 1 << 20, 2 ** 31 - 2)]
    assert all(x >= 0 and x % 256 == 0 for x in sizes) and sizes[0] == 0
    # the largest call there may be
    assert ctx.embed_workspace_bytes(embed_shape(batch=2 ** 15, steps=2 ** 15, per_row=1, dim=1, vocab=2 ** 31 - 2)) > 2 ** 34


# ---- norms, gate and residual sum -----------------------------------------------------------------------------
def residual_shape(**kw):
    d = dict(batch=2, steps=8, dim=64, groups=4, dtype=0, gate_cols=64, gate_act=1, eps_post=1e-5, eps_pre=1e-5, scale_x=1.0, scale_y=1.0)
    d.update(kw)
    return K.PqlResidualShape(*[d[f] for f, _ in K.PqlResidualShape._fields_])


def residual_input(**kw):
    i = K.PqlResidualInput(rows(P), rows(2 * P), rows(3 * P), P, P, None)
    for k, x in kw.items():
        setattr(i, k, x)
    return i


def residual_grad(**kw):
    g = K.PqlResidualGrad(rows(), rows(), rows(), P, P)
    for k, x in kw.items():
        setattr(g, k, x)
    return g


def residual_calls(ctx, s, i=None, total=rows(5 * P), after=rows(6 * P), g=None, ws=P):
    i, g = i or residual_input(), g or residual_grad()
    return (ctx.lib.pql_residual_forward(ctx.h, r(s), r(i), r(total), r(after), None),
            ctx.lib.pql_residual_backward(ctx.h, r(s), r(i), r(total), r(after), r(g), ws, None))


@pytest.mark.parametrize("kw", [dict(batch=-1), dict(steps=-1), dict(batch=1 << 16, steps=1 << 15), dict(dim=0), dict(dim=8193), dict(groups=0),
                                dict(groups=5), dict(dim=514, groups=257), dict(dim=8184, groups=248, gate_cols=0), dict(dim=8190, groups=3, gate_cols=0), dict(dtype=2), dict(gate_cols=2), dict(gate_cols=-1), dict(gate_act=5),
                                dict(gate_act=-1), dict(eps_post=-1e-5), dict(eps_pre=float("nan")), dict(eps_pre=float("inf")),
                                dict(scale_x=float("nan")), dict(scale_y=float("inf"))])
def test_residuals_refuse_bad_shapes(kw):
    ctx, s = K.BlockContext(), residual_shape(**kw)
    assert residual_calls(ctx, s) == (INVALID, INVALID) and ctx.residual_workspace_bytes(s) == INVALID
    assert "bad shape" in ctx.last_error()


def test_residuals_refuse_bad_pointers_and_strides():
    ctx, s = K.BlockContext(), residual_shape()
    both = lambda code, **kw: residual_calls(ctx, s, **kw) == (code, code)  # noqa: E731
    assert residual_calls(ctx, None) == (NULL, NULL) and both(NULL, total=None) and both(NULL, after=None)
    assert both(NULL, i=residual_input(gate=rows(None)))
    assert both(NULL, i=residual_input(x=rows(None), y=rows(None)), g=residual_grad(x=rows(None), y=rows(None), gate=rows(None), post=None))
    assert both(NULL, total=rows(None), after=rows(None), g=residual_grad(pre=None))
    for n in ("x", "y", "gate"):
        assert both(ALIGNMENT, i=residual_input(**{n: rows(P + 2)})) and both(INVALID, i=residual_input(**{n: rows(P, -64)}))
    for n in ("post", "pre", "lengths"):
        assert both(ALIGNMENT, i=residual_input(**{n: P + 2}))
    assert both(ALIGNMENT, total=rows(P + 2)) and both(ALIGNMENT, after=rows(P + 2))
    assert residual_calls(ctx, s, total=rows(P, 63))[0] == INVALID
    # in an input's place, with another stride
    assert residual_calls(ctx, s, total=rows(P, 128))[0] == INVALID and residual_calls(ctx, s, after=rows(2 * P, 128))[0] == INVALID
    back = lambda **kw: residual_calls(ctx, s, total=rows(5 * P, 0), **kw)[1]  # noqa: E731
    assert ctx.lib.pql_residual_backward(ctx.h, r(s), r(residual_input()), r(rows()), r(rows()), None, P, None) == NULL
    assert back(ws=None) == NULL and back(ws=P + 64) == ALIGNMENT
    for n in ("x", "y", "gate"):
        assert back(g=residual_grad(**{n: rows(P + 1, 64)})) == ALIGNMENT
        assert back(g=residual_grad(**{n: rows(9 * P, 63)})) == INVALID
    for n in ("post", "pre"):
        assert back(g=residual_grad(**{n: P + 2})) == ALIGNMENT
    assert back(g=residual_grad(x=rows(5 * P, 64))) == INVALID              # in the place of sum_grad, with another stride
    # gradients of what is not there
    assert back(i=residual_input(x=rows(None))) == INVALID and back(i=residual_input(y=rows(None))) == INVALID
    assert residual_calls(ctx, s, after=rows(None))[1] == INVALID
    s0 = residual_shape(gate_cols=0)
    assert residual_calls(ctx, s0)[1] == INVALID


def test_residual_workspaces():
    ctx = K.BlockContext()
    for dim, groups in ((1, 1), (64, 4), (8192, 1), (8192, 256), (7936, 248), (2304, 256)):
        for batch in (0, 1, 1000, 1 << 20):
            size = ctx.residual_workspace_bytes(residual_shape(batch=batch, dim=dim, groups=groups, gate_cols=0))
            assert 0 <= size <= 8 * 1024 * dim + 256 and size % 256 == 0


# ---- the binding ------------------------------------------------------------------------------------------------
def test_binding_refuses_tensors_that_do_not_fit():
    import torch
    z = lambda *s, dt=torch.float32: torch.zeros(s, dtype=dt)  # noqa: E731
    ctx = K.BlockContext()
    for bad in (z(4), z(2, 2, 2, 2), z(4, 6).t(), z(3, 8, 6)[:, :4], z(3, 8, 6).transpose(0, 1)):
        with pytest.raises(ValueError):
            K.Rows(bad)
    with pytest.raises(TypeError):
        K.Rows(z(4, 6).half())
    assert K.Rows(z(3, 8, 6)[..., 2:5]).c.stride == 6 and K.Rows(z(3, 8, 6)[:, 1:2]).c.stride == 48 and K.Rows(z(5, 6)[2:3]).c.stride == 6
    tokens, table, out = z(2, 3, 4, dt=torch.int32), z(9, 6), z(2, 3, 6)
    s = K.embed_shape(tokens, table, 1.0)
    good = dict(tokens=tokens, lengths=None, table=K.Rows(table), out=K.Rows(out))
    for bad in (dict(tokens=tokens.long()), dict(tokens=tokens[:1]), dict(lengths=z(2)), dict(lengths=z(3, dt=torch.int32)),
                dict(table=K.Rows(z(8, 6))), dict(table=K.Rows(table.bfloat16())), dict(out=K.Rows(z(2, 3, 5))), dict(tokens=tokens.transpose(0, 1))):
        a = {**good, **bad}
        with pytest.raises(ValueError):
            ctx.pql_embed_forward(s, a["tokens"], a["lengths"], a["table"], a["out"], 0)
        with pytest.raises(ValueError):
            ctx.pql_embed_backward(s, a["tokens"], a["lengths"], a["out"], a["table"], None, 0)
    s = K.residual_shape(2, 3, 8, torch.float32, 2, 2, "silu", 1e-5, 1e-5)
    good = dict(x=z(2, 3, 8), y=z(2, 3, 8), gate=z(2, 3, 2), post=z(8), pre=z(8))
    given = K.ResidualInput(s, **good)
    for bad in (dict(x=z(2, 3, 7)), dict(y=z(2, 2, 8)), dict(gate=z(2, 3, 8)), dict(post=z(7)), dict(pre=z(8).bfloat16()), dict(x=z(2, 3, 8).bfloat16()),
                dict(lengths=z(2, dt=torch.int64))):
        with pytest.raises(ValueError):
            K.ResidualInput(s, **{**good, **bad})
    other = K.residual_shape(2, 3, 8, torch.float32, 2, 2, "gelu", 1e-5, 1e-5)
    with pytest.raises(ValueError):
        ctx.pql_residual_forward(other, given, K.Rows(z(2, 3, 8)), None, 0)
    with pytest.raises(ValueError):
        ctx.pql_residual_forward(s, given, K.Rows(z(2, 3, 7)), None, 0)
    with pytest.raises(ValueError):
        ctx.pql_residual_backward(s, given, K.Rows(z(2, 3, 8)), None, K.ResidualGrad(other), None, 0)
    with pytest.raises(TypeError):
        K.residual_shape(2, 3, 8, torch.float16)


def test_empty_calls_do_nothing():
    ctx = K.BlockContext()
    for kw in (dict(batch=0), dict(steps=0)):
        none = rows(None, 0)
        assert ctx.lib.pql_embed_forward(ctx.h, r(embed_shape(**kw)), None, None, r(none), r(none), None) == 0
        s = residual_shape(**kw)
        i = K.PqlResidualInput(none, none, none, None, None, None)
        assert ctx.lib.pql_residual_forward(ctx.h, r(s), r(i), r(none), r(none), None) == 0
        assert ctx.lib.pql_residual_backward(ctx.h, r(s), r(i), r(none), r(none), r(K.PqlResidualGrad(none, none, none, None, None)), None, None) == 0


# ---- the reference's gradients against differences ----------------------------------------------------------------
def differences(f, x, h=1e-5):
    g = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        keep = x[i]
        x[i] = keep + h
        up = f()
        x[i] = keep - h
        down = f()
        x[i] = keep
        g[i] = (up - down) / (2 * h)
    return g


@pytest.mark.parametrize("act", ["none", "sigmoid", "silu", "gelu", "relu"])
def test_activations_of_the_reference(act):
    x = np.linspace(-6, 6, 49) + 0.01
    f, d = O.activate(act, x)
    assert np.allclose(d, (O.activate(act, x + 1e-6)[0] - O.activate(act, x - 1e-6)[0]) / 2e-6, atol=1e-8)


def test_embedding_gradient_of_the_reference():
    rng = np.random.default_rng(0)
    tokens, table, w = rng.integers(-1, 8, (3, 4, 2)), rng.standard_normal((7, 5)), rng.standard_normal((3, 4, 5))
    for lengths in (None, [4, 0, 2]):
        loss = lambda: (w * O.embed(tokens, table, 1.5, lengths)).sum()  # noqa: E731
        assert np.allclose(O.embed_grad(tokens, 7, 1.5, w, lengths), differences(loss, table), atol=1e-8)


@pytest.mark.parametrize("groups,gate,act,eps,form,lengths", [
    (1, 6, "sigmoid", (1e-2, 1e-2), "both", None), (3, 6, "silu", (1e-2, 1e-2), "both", [3, 0]), (2, 2, "gelu", (1e-2, 0.0), "both", [1, 3]),
    (2, 6, "silu", (1e-2, 1e-2), "after", None), (1, 0, "none", (0.0, 1e-2), "before", [2, 3]), (1, 0, "none", (0.0, 0.0), "both", None)])
def test_residual_gradients_of_the_reference(groups, gate, act, eps, form, lengths):
    rng = np.random.default_rng(1)
    n = lambda *s: rng.standard_normal(s)  # noqa: E731
    t = dict(x=n(2, 3, 6) if form != "after" else None, y=n(2, 3, 6) if form != "before" else None,
             gate=n(2, 3, gate) if gate and form != "before" else None, post=n(6), pre=n(6))
    ws, wn = n(2, 3, 6), n(2, 3, 6)
    made = lambda: O.Residual(*t.values(), groups, act, *eps, 0.8, -0.6, lengths)  # noqa: E731
    loss = lambda: (ws * made().sum).sum() + (wn * made().next).sum()  # noqa: E731
    for k, g in made().grad(ws, wn).items():
        if g is not None:
            assert np.allclose(g, differences(loss, t[k]), atol=1e-7), k


@pytest.mark.parametrize("act,lengths", [("silu", None), ("gelu", [2, 0]), ("relu", [1, 3]), ("none", None)])
def test_feed_forward_gradients_of_the_reference(act, lengths):
    rng = np.random.default_rng(2)
    n = lambda *s: rng.standard_normal(s)  # noqa: E731
    t, w = dict(x=n(2, 3, 4), gate=n(5, 4), up=n(5, 4), down=n(4, 5)), n(2, 3, 4)
    real = O.counted((2, 3), lengths)
    loss = lambda: (O.only(w, real) * O.ffn(*t.values(), act, lengths)).sum()  # noqa: E731
    for k, g in O.ffn_grad(*t.values(), act, w, lengths).items():
        assert np.allclose(g, differences(loss, t[k]), atol=1e-7), k


# ---- gated feed-forward block -----------------------------------------------------------------------------------------
def ffn_shape(**kw):
    d = dict(batch=2, steps=8, dim=64, hidden=64, dtype=0, act=2)
    d.update(kw)
    return K.PqlFfnShape(*[d[f] for f, _ in K.PqlFfnShape._fields_])


def ffn_input(**kw):
    i = K.PqlFfnInput(rows(), rows(), rows(), rows(), None)
    for k, x in kw.items():
        setattr(i, k, x)
    return i


def ffn_calls(ctx, s, i=None, out=rows(5 * P), g=None, saved=None, ws=P):
    i, g = i or ffn_input(), g or K.PqlFfnGrad(*[rows()] * 4)
    return (ctx.lib.pql_ffn_forward(ctx.h, r(s), r(i), r(out), saved, ws, None),
            ctx.lib.pql_ffn_backward(ctx.h, r(s), r(i), saved, r(out), r(g), ws, None))


@pytest.mark.parametrize("kw", [dict(batch=-1), dict(steps=-1), dict(batch=1 << 15, steps=1 << 15), dict(dim=0), dict(dim=65537), dict(hidden=0),
                                dict(hidden=65537), dict(dtype=2), dict(act=-1), dict(act=5)])
def test_feed_forward_blocks_refuse_bad_shapes(kw):
    ctx, s = K.BlockContext(), ffn_shape(**kw)
    assert ffn_calls(ctx, s) == (INVALID, INVALID) and ctx.ffn_saved_bytes(s) == INVALID
    assert all(ctx.ffn_workspace_bytes(s, c) == INVALID for c in range(3))
    assert "bad shape" in ctx.last_error()


def test_feed_forward_blocks_refuse_bad_pointers_and_strides():
    ctx, s = K.BlockContext(), ffn_shape()
    both = lambda code, **kw: ffn_calls(ctx, s, **kw) == (code, code)  # noqa: E731
    assert ffn_calls(ctx, None) == (NULL, NULL) and both(NULL, out=None) and both(NULL, out=rows(None)) and both(NULL, ws=None)
    for n in ("x", "gate", "up", "down"):
        assert both(NULL, i=ffn_input(**{n: rows(None)})) and both(ALIGNMENT, i=ffn_input(**{n: rows(P + 2)}))
        assert both(INVALID, i=ffn_input(**{n: rows(P, -64)}))
    assert both(ALIGNMENT, i=ffn_input(lengths=P + 2)) and both(ALIGNMENT, out=rows(P + 2)) and both(ALIGNMENT, ws=P + 128) and both(ALIGNMENT, saved=P + 16)
    assert ffn_calls(ctx, s, out=rows(stride=63))[0] == INVALID
    assert ctx.lib.pql_ffn_backward(ctx.h, r(s), r(ffn_input()), None, r(rows()), None, P, None) == NULL
    for n in ("x", "gate", "up", "down"):
        for bad, code in ((rows(P + 2), ALIGNMENT), (rows(P, 63), INVALID)):
            g = K.PqlFfnGrad(*[rows()] * 4)
            setattr(g, n, bad)
            assert ffn_calls(ctx, s, g=g)[1] == code
    assert ctx.ffn_workspace_bytes(s, 3) == INVALID and ctx.ffn_workspace_bytes(s, -1) == INVALID
    none = rows(None, 0)
    for kw in (dict(batch=0), dict(steps=0)):
        e = ffn_shape(**kw)
        assert ctx.lib.pql_ffn_forward(ctx.h, r(e), r(K.PqlFfnInput(none, none, none, none, None)), r(none), None, None, None) == 0


def test_feed_forward_workspaces():
    ctx = K.BlockContext()
    for kw in (dict(), dict(batch=0), dict(dim=1, hidden=1), dict(dtype=1), dict(batch=1 << 14, dim=4096, hidden=65536)):
        s = ffn_shape(**kw)
        sizes = [ctx.ffn_workspace_bytes(s, c) for c in (K.FFN_FORWARD, K.FFN_BACKWARD, K.FFN_BACKWARD_ALONE)]
        assert all(x >= 0 and x % 256 == 0 for x in sizes)
        assert sizes[2] == sizes[1] + ctx.ffn_saved_bytes(s)


def test_binding_refuses_matrices_that_do_not_fit():
    import torch
    z = lambda *s, dt=torch.float32: torch.zeros(s, dtype=dt)  # noqa: E731
    ctx, x, w, down = K.BlockContext(), z(2, 3, 8), z(12, 8), z(8, 12)
    s = K.ffn_shape(x, w, "silu")
    good = dict(x=x, gate=w, up=w, down=down)
    given = K.FfnInput(s, **good)
    for bad in (dict(x=z(2, 3, 7)), dict(x=z(3, 3, 8)), dict(gate=z(11, 8)), dict(up=z(12, 8).bfloat16()), dict(down=w), dict(lengths=z(3, dt=torch.int32))):
        with pytest.raises(ValueError):
            K.FfnInput(s, **{**good, **bad})
    other = K.ffn_shape(x, w, "gelu")
    with pytest.raises(ValueError):
        ctx.pql_ffn_forward(other, given, K.Rows(z(2, 3, 8)), None, None, 0)
    with pytest.raises(ValueError):
        ctx.pql_ffn_forward(s, given, K.Rows(z(2, 3, 7)), None, None, 0)
    with pytest.raises(ValueError):
        ctx.pql_ffn_backward(s, given, None, K.Rows(z(2, 3, 8)), K.FfnGrad(other), None, 0)
    for bad in ((z(2, 8), w), (x, z(12, 7)), (x, w.bfloat16())):
        with pytest.raises(ValueError):
            K.ffn_shape(*bad, "silu")


# ---- what a call is refused for: arguments that fit get as far as the check of the device, which tensors of the host do not pass ----
AWAY = "tensors of another device"


def blocks(torch):
    """A call of each kind on tensors of the host, as (function of its arguments, arguments that fit, memory that it needs)."""
    ctx = K.BlockContext()
    z = lambda *s, dt=torch.float32: torch.zeros(s, dtype=dt)  # noqa: E731
    space = lambda n: torch.zeros(n, dtype=torch.uint8)  # noqa: E731
    tokens, table, out = z(2, 3, 4, dt=torch.int32), z(9, 6), z(2, 3, 6)
    es = K.embed_shape(tokens, table, 1.0)
    rs = K.residual_shape(2, 3, 8, torch.float32, 2, 2, "silu", 1e-5, 1e-5)
    given = K.ResidualInput(rs, z(2, 3, 8), z(2, 3, 8), z(2, 3, 2), z(8), z(8))
    fs = K.ffn_shape(z(2, 3, 8), z(12, 8), "silu")
    f = K.FfnInput(fs, z(2, 3, 8), z(12, 8), z(12, 8), z(8, 12))
    need = [ctx.ffn_workspace_bytes(fs, c) for c in range(3)]
    x = lambda: K.Rows(z(2, 3, 8))  # noqa: E731
    return z, space, [
        (ctx.pql_embed_forward, dict(shape=es, tokens=tokens, lengths=None, table=K.Rows(table), out=K.Rows(out)), {}),
        (ctx.pql_embed_backward, dict(shape=es, tokens=tokens, lengths=None, out_grad=K.Rows(out), table_grad=K.Rows(table),
                                      workspace=space(ctx.embed_workspace_bytes(es))), dict(workspace=ctx.embed_workspace_bytes(es))),
        (ctx.pql_residual_forward, dict(shape=rs, given=given, sum=x(), next=x()), {}),
        (ctx.pql_residual_backward, dict(shape=rs, given=given, sum_grad=x(), next_grad=x(), grads=K.ResidualGrad(rs, post=z(8)),
                                         workspace=space(ctx.residual_workspace_bytes(rs))), dict(workspace=ctx.residual_workspace_bytes(rs))),
        (ctx.pql_ffn_forward, dict(shape=fs, given=f, out=x(), saved=space(ctx.ffn_saved_bytes(fs)), workspace=space(need[0])),
         dict(saved=ctx.ffn_saved_bytes(fs), workspace=need[0])),
        (ctx.pql_ffn_backward, dict(shape=fs, given=f, saved=space(ctx.ffn_saved_bytes(fs)), out_grad=x(), grads=K.FfnGrad(fs), workspace=space(need[1])),
         dict(saved=ctx.ffn_saved_bytes(fs), workspace=need[1])),
        (ctx.pql_ffn_backward, dict(shape=fs, given=f, saved=None, out_grad=x(), grads=K.FfnGrad(fs), workspace=space(need[2])), dict(workspace=need[2])),
    ]


def refused(call, args, match, **bad):
    with pytest.raises(ValueError, match=match):
        call(**{**args, **bad}, stream=0)


def test_binding_refuses_memory_that_is_too_small():
    import torch
    _, space, calls = blocks(torch)
    for call, args, need in calls:
        refused(call, args, AWAY)
        for name, size in need.items():
            assert size > 0
            refused(call, args, "%s: expected at least %d contiguous bytes, got %d" % (name, size, size - 1), **{name: space(size - 1)})
            refused(call, args, name + ": expected at least", **{name: space(2 * size)[::2]})
            refused(call, args, AWAY, **{name: space(size + 8)[8:]})
    # one shape, three sizes: what is enough with saved is not without
    call, args, need = calls[-1]
    refused(call, args, "workspace: expected at least", workspace=calls[-2][1]["workspace"])
    # no gradient of a weight: no workspace is used
    call, args, _ = calls[3]
    refused(call, args, AWAY, workspace=space(1), grads=K.ResidualGrad(args["shape"]))


def test_binding_refuses_calls_by_what_does_not_fit():
    """Each refusal by its own message; what fits is refused for its device alone."""
    import torch
    z, space, calls = blocks(torch)
    e, er = calls[0], calls[1]
    tokens, table = e[1]["tokens"], torch.zeros(9, 6)
    for bad, match in ((dict(tokens=tokens.long()), "tokens: expected a contiguous int32 tensor of 24"), (dict(tokens=tokens[:1]), "tokens: expected"),
                       (dict(tokens=tokens.transpose(0, 1)), "tokens: expected a contiguous"), (dict(lengths=z(2)), "lengths: expected a contiguous int32"),
                       (dict(lengths=z(3, dt=torch.int32)), "lengths: expected a contiguous int32 tensor of 2")):
        refused(e[0], e[1], match, **bad)
        refused(er[0], er[1], match, **bad)
    for bad in (K.Rows(z(8, 6)), K.Rows(table.bfloat16()), K.Rows(z(9, 5))):
        refused(e[0], e[1], "table: 9 rows of 6 \\(type 0\\) expected", table=bad)
        refused(er[0], er[1], "table: 9 rows of 6 \\(type 0\\) expected", table_grad=bad)
    for bad in (K.Rows(z(2, 3, 5)), K.Rows(z(2, 4, 6)), K.Rows(z(2, 3, 6).bfloat16())):
        refused(e[0], e[1], "rows: 6 rows of 6 \\(type 0\\) expected", out=bad)
        refused(er[0], er[1], "rows: 6 rows of 6 \\(type 0\\) expected", out_grad=bad)
    x, narrow = K.Rows(z(2, 3, 8)), K.Rows(z(2, 3, 7))
    other = K.residual_shape(2, 3, 8, torch.float32, 2, 2, "gelu", 1e-5, 1e-5)
    for call, args, _ in calls[2:4]:
        refused(call, args, "do not agree", shape=other)
        refused(call, args, "do not agree", given=K.ResidualInput(other, z(2, 3, 8), z(2, 3, 8), z(2, 3, 2)))
    refused(*calls[3][:2], "do not agree", grads=K.ResidualGrad(other))
    for names, (call, args, _) in zip((("sum", "next"), ("sum_grad", "next_grad")), calls[2:4]):
        for name in names:
            refused(call, args, name + ": 6 rows of 8", **{name: narrow})
            refused(call, args, name + ": 6 rows of 8", **{name: K.Rows(z(2, 3, 8).bfloat16())})
            refused(call, args, AWAY, **{name: None})
    other = K.ffn_shape(z(2, 3, 8), z(12, 8), "gelu")
    away = K.FfnInput(other, z(2, 3, 8), z(12, 8), z(12, 8), z(8, 12))
    for call, args, _ in calls[4:]:
        refused(call, args, "do not agree", shape=other)
        refused(call, args, "do not agree", given=away)
        name = "out" if "out" in args else "out_grad"
        refused(call, args, name + ": 6 rows of 8", **{name: narrow})
        refused(call, args, AWAY, **{name: x})
        if "grads" in args:
            refused(call, args, "do not agree", grads=K.FfnGrad(other))
    # the descriptions
    rs, fs = calls[2][1]["shape"], calls[4][1]["shape"]
    good = dict(x=z(2, 3, 8), y=z(2, 3, 8), gate=z(2, 3, 2), post=z(8), pre=z(8))
    for bad, match in ((dict(x=z(2, 3, 7)), "x: 6 rows of 8"), (dict(y=z(2, 2, 8)), "y: 6 rows of 8"), (dict(gate=z(2, 3, 8)), "gate: 6 rows of 2"),
                       (dict(post=z(7)), "post: expected a contiguous float32 tensor of 8"), (dict(pre=z(8).bfloat16()), "pre: expected"),
                       (dict(x=z(2, 3, 8).bfloat16()), "x: 6 rows of 8"), (dict(lengths=z(2, dt=torch.int64)), "lengths: expected")):
        with pytest.raises(ValueError, match="ResidualInput: " + match):
            K.ResidualInput(rs, **{**good, **bad})
    good = dict(x=z(2, 3, 8), gate=z(12, 8), up=z(12, 8), down=z(8, 12))
    for bad, match in ((dict(x=z(2, 3, 7)), "x: 6 rows of 8"), (dict(x=z(3, 3, 8)), "x: 6 rows of 8"), (dict(gate=z(11, 8)), "gate: 12 rows of 8"),
                       (dict(up=z(12, 8).bfloat16()), "up: 12 rows of 8"), (dict(down=z(12, 8)), "down: 8 rows of 12"),
                       (dict(lengths=z(3, dt=torch.int32)), "lengths: expected a contiguous int32 tensor of 2")):
        with pytest.raises(ValueError, match="FfnInput: " + match):
            K.FfnInput(fs, **{**good, **bad})
