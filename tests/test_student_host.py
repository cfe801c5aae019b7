"""The student's operators on the host: header, binding, refusals before any launch, and the double-precision
reference's gradients against differences."""
import ctypes as C
import os
import re
import shutil
import subprocess

import numpy as np
import pytest

from oracle import student_oracle as O
from paper_2307_12983_amd import binding as B
from paper_2307_12983_amd import student as S

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "pql_student.h")
P = 0x1000                                      # never dereferenced: validation fails first


def header_text():
    return re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)


def test_library_exports_what_the_header_declares_with_the_bindings_prototypes():
    lib = S.load_library()
    protos = re.findall(r"\b(int32_t|int64_t)\s+(pql_[a-z_]+)\s*\(([^)]*)\)\s*;", header_text())
    assert sorted(n for _, n, _ in protos) == sorted(S.EXPORTS)
    scalars = {"int32_t": C.c_int32, "int64_t": C.c_int64, "float": C.c_float}
    by_value = {"pql_seq": S.PqlSeq, "pql_logits": S.PqlLogits, "pql_teacher": S.PqlTeacher}
    for ret, name, params in protos:
        fn = getattr(lib, name)
        assert fn.restype is scalars[ret], name
        plist = [p.strip() for p in params.split(",")]
        assert len(plist) == len(fn.argtypes), name
        for p, t in zip(plist, fn.argtypes):
            if "*" in p:
                assert t is C.c_void_p or issubclass(t, C._Pointer), (name, p)
            else:
                base = p.split()[0]
                assert t is by_value.get(base, scalars.get(base)), (name, p)


def test_header_is_plain_c_and_the_ctypes_structures_have_its_layout(tmp_path):
    gcc, gxx = shutil.which("gcc"), shutil.which("g++")
    if not gcc or not gxx:
        pytest.skip("no host C compiler")
    for cc, std, lang in ((gcc, "-std=c99", "c"), (gxx, "-std=c++11", "c++")):
        r = subprocess.run([cc, std, "-x", lang, "-Wall", "-Wextra", "-pedantic", "-Werror", "-fsyntax-only", HEADER],
                           capture_output=True, text=True)
        assert r.returncode == 0, r.stderr
    mirrors = {"pql_seq": S.PqlSeq, "pql_delta_shape": S.PqlDeltaShape, "pql_delta_input": S.PqlDeltaInput,
               "pql_delta_grad": S.PqlDeltaGrad, "pql_logits": S.PqlLogits, "pql_teacher": S.PqlTeacher}
    consts = {"PQL_F32": S.PQL_F32, "PQL_BF16": S.PQL_BF16, "PQL_MAX_TOP": S.PQL_MAX_TOP,
              "PQL_DELTA_MAX_DIM_K": S.PQL_DELTA_MAX_DIM_K, "PQL_DELTA_MAX_DIM_V": S.PQL_DELTA_MAX_DIM_V}
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "pql_student.h"', "int main(void) {"]
    for cname, cls in mirrors.items():
        lines.append('printf("%s %%zu\\n", sizeof(%s));' % (cname, cname))
        lines += ['printf("%s.%s %%zu\\n", offsetof(%s, %s));' % (cname, f, cname, f) for f, _ in cls._fields_]
    lines += ['printf("%s %%d\\n", %s);' % (n, n) for n in consts] + ["return 0; }"]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines))
    r = subprocess.run([gcc, "-std=c99", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    got = dict(l.split() for l in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.splitlines())
    for cname, cls in mirrors.items():
        assert int(got[cname]) == C.sizeof(cls), cname
        for f, _ in cls._fields_:
            assert int(got["%s.%s" % (cname, f)]) == getattr(cls, f).offset, "%s.%s" % (cname, f)
    for n, x in consts.items():
        assert int(got[n]) == x


def _shape(**kw):
    d = dict(batch=2, steps=8, heads_k=2, heads_v=4, dim_k=16, dim_v=24, dtype=S.PQL_F32, scale=0.25)
    d.update(kw)
    return S.PqlDeltaShape(*[d[f] for f, _ in S.PqlDeltaShape._fields_])


def _seq(data=P, b=1 << 16, t=1 << 8, h=32):
    return S.PqlSeq(data, b, t, h)


def _input(**kw):
    i = S.PqlDeltaInput(*[_seq()] * 5, None, None)
    for k, x in kw.items():
        setattr(i, k, x)
    return i


@pytest.mark.parametrize("kw", [dict(batch=-1), dict(steps=-1), dict(heads_k=0), dict(heads_v=0), dict(heads_v=3), dict(dim_k=0),
                                dict(dim_k=129), dict(dim_v=0), dict(dim_v=257), dict(dtype=2), dict(scale=float("nan")),
                                dict(heads_v=65536)])
def test_delta_refuses_bad_shapes(kw):
    ctx, s = S.StudentContext(), _shape(**kw)
    lib, i = ctx.lib, _input()
    assert ctx.delta_saved_bytes(s) == -1 and ctx.delta_workspace_bytes(s, True) == -1
    assert lib.pql_delta_step(ctx.h, C.byref(s), C.byref(i), P, _seq(), None) == -1
    assert lib.pql_delta_forward(ctx.h, C.byref(s), C.byref(i), _seq(), P, None, P, None) == -1
    g = S.PqlDeltaGrad(*[_seq()] * 5, None)
    assert lib.pql_delta_backward(ctx.h, C.byref(s), C.byref(i), P, _seq(), None, C.byref(g), P, None) == -1
    assert "bad shape" in ctx.last_error()


def test_delta_refuses_null_misaligned_and_overlapping_pointers():
    ctx, s = S.StudentContext(), _shape()
    lib, r = ctx.lib, C.byref

    def step(i, state=P, out=_seq()):
        return lib.pql_delta_step(ctx.h, r(s), r(i), state, out, None)

    assert lib.pql_delta_step(None, r(s), r(_input()), P, _seq(), None) == -2
    assert lib.pql_delta_step(ctx.h, None, r(_input()), P, _seq(), None) == -2
    for n in ("q", "k", "v", "log_decay", "beta"):
        assert step(_input(**{n: _seq(None)})) == -2
        assert step(_input(**{n: _seq(P + 1)})) == -6
    assert step(_input(state=P + 4)) == -6 and step(_input(lengths=P + 2)) == -6
    assert step(_input(), state=None) == -2 and step(_input(), state=P + 8) == -6
    assert step(_input(), out=_seq(None)) == -2 and step(_input(), out=_seq(P + 2)) == -6
    assert step(_input(), out=_seq(P, h=0)) == -1 and step(_input(), out=_seq(P, t=0)) == -1
    fwd = lambda out=_seq(), state=P, saved=None, ws=P: lib.pql_delta_forward(ctx.h, r(s), r(_input()), out, state, saved, ws, None)  # noqa: E731
    assert fwd(out=_seq(None)) == -2 and fwd(ws=None) == -2 and fwd(ws=P + 16) == -6 and fwd(saved=P + 16) == -6
    assert fwd(state=P + 4) == -6 and fwd(out=_seq(P, b=0)) == -1
    g = S.PqlDeltaGrad(*[_seq()] * 5, None)
    bwd = lambda g=g, saved=P, do=_seq(), ds=None, ws=P: lib.pql_delta_backward(ctx.h, r(s), r(_input()), saved, do, ds, r(g), ws, None)  # noqa: E731
    assert bwd(saved=None) == -2 and bwd(do=_seq(None)) == -2 and bwd(ws=None) == -2
    assert bwd(ws=P + 8) == -6 and bwd(saved=P + 8) == -6 and bwd(ds=P + 8) == -6
    for n in ("q", "k", "v", "log_decay", "beta"):
        x = S.PqlDeltaGrad(*[_seq()] * 5, None)
        setattr(x, n, _seq(None))
        assert bwd(x) == -2
        setattr(x, n, _seq(P, h=0))
        assert bwd(x) == -1
    assert lib.pql_delta_backward(ctx.h, r(s), r(_input()), P, _seq(), None, None, P, None) == -2


def test_empty_calls_do_nothing():
    ctx = S.StudentContext()
    s = _shape(batch=0)
    assert ctx.lib.pql_delta_step(ctx.h, C.byref(s), C.byref(_input()), None, _seq(None), None) == 0
    assert ctx.lib.pql_delta_forward(ctx.h, C.byref(s), C.byref(_input()), _seq(None), None, None, None, None) == 0
    z = S.PqlLogits(None, 0, 64, 64, 0)
    assert ctx.lib.pql_top_logits(ctx.h, z, 4, None, None, None, None) == 0
    assert ctx.lib.pql_distill_loss(ctx.h, z, S.PqlTeacher(None, None, 4), 1.0, None, None, None, S.NO_GRAD, None, None) == 0


def test_rows_refuse_bad_arguments():
    ctx = S.StudentContext()
    lib = ctx.lib
    z = S.PqlLogits(P, 4, 64, 64, 0)
    t = S.PqlTeacher(P, P, 8)
    top = lambda z=z, k=8, i=P, v=P, ws=P: lib.pql_top_logits(ctx.h, z, k, i, v, ws, None)  # noqa: E731
    for bad in (S.PqlLogits(P, -1, 64, 64, 0), S.PqlLogits(P, 4, 63, 64, 0), S.PqlLogits(P, 4, 64, 0, 0), S.PqlLogits(P, 4, 64, 64, 3)):
        assert top(bad) == -1 and lib.pql_top_logits_workspace_bytes(C.byref(bad), 1) == -1
        assert lib.pql_distill_workspace_bytes(C.byref(bad)) == -1
        assert lib.pql_distill_loss(ctx.h, bad, t, 1.0, None, P, P, S.NO_GRAD, P, None) == -1
    for k in (0, 65, 257, -1):
        assert top(k=k) == -1
    assert top(i=None) == -2 and top(v=None) == -2 and top(S.PqlLogits(None, 4, 64, 64, 0)) == -2
    assert top(S.PqlLogits(P + 2, 4, 64, 64, 0)) == -6 and top(i=P + 2) == -6 and top(ws=P + 8) == -6
    few = S.PqlLogits(P, 2, 1 << 17, 1 << 17, 1)
    assert lib.pql_top_logits_workspace_bytes(C.byref(few), 8) > 0 and top(few, ws=None) == -2
    loss = lambda z=z, t=t, temp=1.0, w=None, l=P, e=P, g=S.NO_GRAD, ws=P: lib.pql_distill_loss(ctx.h, z, t, temp, w, l, e, g, ws, None)  # noqa: E731
    for temp in (0.0, -1.0, float("nan"), float("inf"), 1e-39):
        assert loss(temp=temp) == -1
    for k in (0, 65, 257):
        assert loss(t=S.PqlTeacher(P, P, k)) == -1
    assert loss(t=S.PqlTeacher(None, P, 8)) == -2 and loss(t=S.PqlTeacher(P, None, 8)) == -2
    assert loss(l=None) == -2 and loss(e=None) == -2 and loss(w=P + 1) == -6 and loss(l=P + 2) == -6
    for g in (S.PqlLogits(P, 3, 64, 64, 0), S.PqlLogits(P, 4, 64, 63, 0), S.PqlLogits(P, 4, 64, 64, 1), S.PqlLogits(P, 4, 60, 64, 0),
              S.PqlLogits(P, 4, 80, 64, 0)):               # the last one: in the logits' place with another stride
        assert loss(g=g) == -1
        assert lib.pql_distill_backward(ctx.h, z, t, 1.0, P, P, g, None) == -1
    assert loss(few, ws=None) == -2
    back = lambda e=P, c=P, g=z: lib.pql_distill_backward(ctx.h, z, t, 1.0, e, c, g, None)  # noqa: E731
    assert back(e=None) == -2 and back(c=None) == -2 and back(g=S.PqlLogits(None, 4, 64, 64, 0)) == -2 and back(c=P + 2) == -6


def test_saved_and_workspace_sizes():
    ctx = S.StudentContext()
    for kw in (dict(), dict(steps=64), dict(steps=65), dict(heads_v=2), dict(dim_k=128, dim_v=200), dict(steps=0)):
        s = _shape(**kw)
        saved, fwd, bwd = ctx.delta_saved_bytes(s), ctx.delta_workspace_bytes(s, False), ctx.delta_workspace_bytes(s, True)
        assert all(x >= 0 and x % 256 == 0 for x in (saved, fwd, bwd)) and bwd >= fwd
    assert ctx.delta_saved_bytes(_shape(steps=65)) > ctx.delta_saved_bytes(_shape(steps=64))


def test_binding_refuses_tensors_that_do_not_fit():
    import torch
    z = lambda *s, dt=torch.float32: torch.zeros(s, dtype=dt)  # noqa: E731
    q, v, g = z(2, 8, 2, 16), z(2, 8, 4, 24), z(2, 8, 4)
    S.DeltaInput(q, q, v, g, g, torch.zeros(2, dtype=torch.int32), z(2, 4, 16, 24))
    for bad in (dict(k=z(2, 8, 2, 15)), dict(k=q.bfloat16()), dict(log_decay=g.double()), dict(beta=z(2, 8, 2)),
                dict(lengths=torch.zeros(2, dtype=torch.int64)), dict(lengths=torch.zeros(3, dtype=torch.int32)),
                dict(state=z(2, 4, 24, 16)), dict(q=q.transpose(2, 3))):
        kw = dict(q=q, k=q, v=v, log_decay=g, beta=g)
        kw.update(bad)
        with pytest.raises(ValueError):
            S.DeltaInput(**kw)
    with pytest.raises(TypeError):
        S.delta_shape(q.half(), v.half(), 1.0)
    with pytest.raises(ValueError):
        S.Logits(z(3, 5).t())
    with pytest.raises(ValueError):
        S.Teacher(torch.zeros(2, 3, dtype=torch.int64), z(2, 3))


# ---- the reference itself ---------------------------------------------------------------------
def _differences(f, x, eps=1e-6):
    g = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        if not np.isfinite(x[i]):
            continue
        old = x[i]
        x[i] = old + eps
        up = f()
        x[i] = old - eps
        g[i] = (up - f()) / (2 * eps)
        x[i] = old
    return g


def test_reference_gradients_of_the_delta_rule_agree_with_differences():
    rng = np.random.default_rng(3)
    n, t, hk, hv, dk, dv = 2, 5, 1, 2, 3, 2
    q, k = rng.standard_normal((2, n, t, hk, dk)) * 0.6
    v = rng.standard_normal((n, t, hv, dv))
    g = -rng.random((n, t, hv))
    g[0, 2, 1] = -np.inf
    beta = rng.random((n, t, hv)) * 1.5
    state, lengths = rng.standard_normal((n, hv, dk, dv)), [5, 3]
    do, ds = rng.standard_normal((n, t, hv, dv)), rng.standard_normal((n, hv, dk, dv))

    def loss():
        out, s = O.delta_forward(q, k, v, g, beta, 0.7, lengths, state)
        return np.sum(out * do) + np.sum(s * ds)

    got = O.delta_backward(q, k, v, g, beta, 0.7, do, ds, lengths, state)
    for x, d in zip((q, k, v, g, beta, state), got):
        want = _differences(loss, x)
        # central differences: step^2 truncation and 1e-16 / step rounding, both below 1e-8 at values of order one
        assert np.max(np.abs(d - want)) < 1e-7


def test_reference_gradient_of_the_distillation_agrees_with_differences():
    rng = np.random.default_rng(4)
    z = rng.standard_normal((4, 6))
    z[1, 2] = -np.inf
    index = np.array([[0, 3, -1], [1, 4, 5], [2, 2, 9], [-1, -1, 7]])
    value, weight = rng.standard_normal((4, 3)), np.array([0.5, 1.0, 2.0, 1.0])
    loss, _, grad = O.distill(z, index, value, 1.7, weight)
    assert loss[3] == 0 and not grad[3].any()
    want = _differences(lambda: float(np.sum(O.distill(z, index, value, 1.7, weight)[0])), z)
    assert np.max(np.abs(grad - want)) < 1e-7


def test_calls_refuse_tensors_that_do_not_belong_together():
    """Before anything is launched: the kernels take sizes from the logits or the shape alone."""
    import torch
    ctx = S.StudentContext()
    z = lambda *s, dt=torch.float32: torch.zeros(s, dtype=dt)  # noqa: E731
    rows, vocab, top = 6, 40, 4
    logits, lists = S.Logits(z(rows, vocab)), lambda n: S.Teacher(z(n, top, dt=torch.int32), z(n, top))  # noqa: E731
    for i, v in ((z(rows - 1, top, dt=torch.int32), z(rows, top)), (z(rows, top, dt=torch.int64), z(rows, top)), (z(rows, top), z(rows, top)),
                 (z(rows, top, dt=torch.int32), z(rows, top + 1)), (z(rows, top, dt=torch.int32), z(rows, top, dt=torch.bfloat16)),
                 (z(rows, top, dt=torch.int32), z(top, rows).t())):
        with pytest.raises(ValueError):
            ctx.pql_top_logits(logits, top, i, v, None)
    good = dict(teacher=lists(rows), row_weight=None, loss=z(rows), lse=z(rows))
    for bad in (dict(teacher=lists(rows - 1)), dict(row_weight=z(rows - 1)), dict(loss=z(1)), dict(lse=z(rows, dt=torch.float64)), dict(loss=z(2 * rows)[::2])):
        a = {**good, **bad}
        with pytest.raises(ValueError):
            ctx.pql_distill_loss(logits, a["teacher"], 1.0, a["row_weight"], a["loss"], a["lse"], None, None)
        if "row_weight" not in bad:
            with pytest.raises(ValueError):
                ctx.pql_distill_backward(logits, a["teacher"], 1.0, a["lse"], a["loss"], logits)
    q, v, g = z(2, 8, 2, 16), z(2, 8, 4, 24), z(2, 8, 4)
    shape, given, out = S.delta_shape(q, v, 0.25), S.DeltaInput(q, q, v, g, g), S.Sequence(z(2, 8, 4, 24))
    grads = S.DeltaGrad(z(2, 8, 2, 16), z(2, 8, 2, 16), z(2, 8, 4, 24), z(2, 8, 4), z(2, 8, 4))
    for state in (z(2, 4, 24, 16), z(1, 4, 16, 24), z(2, 4, 16, 24, dt=torch.bfloat16), z(2, 4, 24, 16).transpose(2, 3)):
        with pytest.raises(ValueError):
            ctx.pql_delta_step(shape, given, state, out)
        with pytest.raises(ValueError):
            ctx.pql_delta_forward(shape, given, out, state, None, None)
        with pytest.raises(ValueError):
            ctx.pql_delta_backward(shape, given, None, out, state, grads, None)
    for wrong in (z(2, 8, 4, 23), z(2, 8, 4, 24, dt=torch.bfloat16), z(2, 7, 4, 24)):
        with pytest.raises(ValueError):
            ctx.pql_delta_step(shape, given, None, S.Sequence(wrong))


def test_rows_are_walked_beyond_32_bits_of_elements(tmp_path):
    """The walk over rows behind a sequence's length, on the host: 2^27 rows of 16 columns are 2^31 elements."""
    from paper_2307_12983_amd import build
    src, exe = tmp_path / "rows.hip", tmp_path / "rows"
    src.write_text("""
#include <cstdio>
#include "pql_student_internal.h"
template <int COLS> void walk(int64_t from, int64_t to, int n) {
    int64_t seen = 0, first = to, last = -1, bad = 0;
    for (int lane = 0; lane < 64; lane += lane == 0 ? 1 : 62)        // lanes 0, 1 and 63
        pql::each_of_rows<COLS>(lane, from, to, n, [&](int64_t row, int c) {
            ++seen; first = row < first ? row : first; last = row > last ? row : last; bad += c != lane % COLS || c >= n;
        });
    printf("%lld %lld %lld %lld\\n", (long long)seen, (long long)first, (long long)last, (long long)bad);
}
int main() { walk<16>(3, 3 + (1ll << 27), 16); walk<32>(0, 7, 20); walk<32>(5, 5, 32); return 0; }
""")
    r = subprocess.run([build._hipcc(), "-O1", "-std=c++17", "--offload-arch=gfx950", "--offload-host-only", "-I" + build.CSRC,
                        "-I" + os.path.join(ROOT, "include"), str(src), "-o", str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    got = [[int(x) for x in l.split()] for l in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.splitlines()]
    quarter = 2 ** 25
    assert got == [[3 * quarter, 3, 2 + 2 ** 27, 0], [4 + 4, 0, 6, 0], [0, 5, -1, 0]]
