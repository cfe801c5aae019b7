"""The student's operators where values, sizes or counts come to the limits of what the calls take, against the
double-precision reference.  Tolerances: those of test_gpu_student.py, derived there."""
import numpy as np
import pytest

from test_gpu_student import NORM, Delta, close, env, lists, logits  # noqa: F401

pytestmark = pytest.mark.gpu
GRADS = ("dq", "dk", "dv", "dg", "dbeta", "dstate")
LOWEST = float(np.finfo(np.float32).min)


def held(x):
    """What 32 bits hold of a value: nothing below half their smallest number, infinity from 2^128 on."""
    x = np.where(np.abs(x) < 2.0 ** -150, 0.0, x)
    return np.where(np.abs(x) >= 2.0 ** 128, np.copysign(np.inf, x), x)


def set_gate(d, places, value):
    for b, i in places:
        d.g[b, i] = value
        d.host[3][b, i] = float(np.float32(value))


# chunks of 32 and of 64 tokens, rows with and without 16-byte granules
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("size", [(2, 96, 1, 2, 32, 40), (2, 70, 2, 2, 33, 20), (1, 577, 1, 2, 128, 96), (1, 577, 1, 1, 20, 17)])
@pytest.mark.parametrize("value", [-60.0, -110.0, -1e9, -1e12, -1e30, LOWEST])
def test_finite_decays_that_leave_nothing(env, size, dtype, value):
    """A decay far below what 32 bits can hold, at the start, inside and at the end of chunks: what follows it
    depends on the gates behind it alone."""
    t = size[1]
    d = Delta(env, *size, dtype=dtype, seed=t)
    set_gate(d, [(0, i) for i in (0, 5, 31, 32, 45, 63, 64, t - 1)], value)
    out, state = d.want()
    for name, got in (("step", d.step()), ("forward", d.forward())):
        close(got[0], out, name + " out")
        close(got[1], state, name + " state")
    for name, got, want in zip(GRADS, d.backward(d.forward(True)[2]), d.want_grads()):
        close(got, held(want), name)


# ---- values that are not finite ----------------------------------------------------------------
# An episode from token 5 to 11 or, for states, from the start to 11; good ones around it, in the same chunks.
POISON = ["state inf", "state nan", "v inf", "v nan", "k nan", "k inf", "q nan", "beta nan", "decay nan"]


def poisoned(env, size, dtype, kind, layout="dense"):
    torch = env[0]
    t = size[1]
    whole = kind.startswith("state")
    d = Delta(env, *size, dtype=dtype, layout=layout, resets=[(0, i) for i in ((12, 40, 64, t - 2) if whole else (5, 12, 40, 64, t - 2))], seed=t + 1)
    what, value = kind.split()
    value = float(value)
    if whole:
        d.state[0, 0, 1, 2] = value
        d.host_state[0, 0, 1, 2] = value
    else:
        at = {"v": (0, 7, 0, 2), "k": (0, 7, 0, 1), "q": (0, 7, 0, 1), "beta": (0, 7, 0), "decay": (0, 7, 0)}[what]
        i = ["q", "k", "v", "decay", "beta"].index(what)
        (d.q, d.k, d.v, d.g, d.beta)[i][at] = value
        d.host[i][at] = value
    torch.cuda.synchronize()
    return d, (range(0, 12) if whole else range(5, 12))


SICK = [(2, 70, 1, 2, 32, 40), (2, 70, 1, 1, 128, 24), (64, 66, 2, 4, 20, 36), (64, 66, 2, 4, 72, 64), (1, 577, 1, 1, 64, 20), (1, 577, 1, 2, 128, 33)]


@pytest.mark.parametrize("kind", POISON)
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("size", SICK)
@pytest.mark.filterwarnings("ignore:invalid value:RuntimeWarning")
def test_values_that_are_not_finite_stay_in_their_episode(env, size, dtype, kind):
    """Both forms give what the recurrence gives: finite wherever that is, in other episodes of the same chunk and
    before the value, and gradients of all other episodes as if there were none."""
    d, bad = poisoned(env, size, dtype, kind)
    out, state = d.want()
    kept = d.forward(True)
    for name, got in (("step", d.step()), ("forward", d.forward()), ("forward, kept", kept[:2])):
        for part, x, y in zip((" out", " state"), got, (out, state)):
            host, fine = x.double().cpu().numpy(), np.isfinite(y)
            assert np.array_equal(np.isfinite(host), fine), name + part + ": finite in other places than the recurrence's"
            close(x[torch_mask(x, fine)], y[fine], name + part)
    good = np.ones(size[1], bool)
    good[list(bad)] = False
    want = d.want_grads()
    grads = d.backward(kept[2])
    for name, x, y in zip(GRADS[:5], grads, want):
        assert np.isfinite(y[:, good]).all(), name
        close(x[:, torch_mask(x, good)], y[:, good], name)
    fine = np.isfinite(want[5])
    if not kind.startswith("state"):
        assert fine.all()
    close(grads[5][torch_mask(grads[5], fine)], want[5][fine], "dstate")


def torch_mask(x, mask):
    import torch
    return torch.from_numpy(np.ascontiguousarray(mask)).to(x.device)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("layout", ["offset", "packed"])
@pytest.mark.filterwarnings("ignore:invalid value:RuntimeWarning")
def test_values_that_are_not_finite_in_other_layouts(env, layout, dtype):
    d, bad = poisoned(env, (2, 70, 1, 2, 33, 20), dtype, "v nan", layout)
    out, state = d.want()
    got = d.forward(True)
    fine = np.isfinite(out)
    assert np.array_equal(np.isfinite(got[0].double().cpu().numpy()), fine)
    close(got[0][torch_mask(got[0], fine)], out[fine], "out")
    close(got[1], state, "state")
    good = np.ones(70, bool)
    good[list(bad)] = False
    for name, x, y in zip(GRADS[:5], d.backward(got[2]), d.want_grads()):
        close(x[:, torch_mask(x, good)], y[:, good], name)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.filterwarnings("ignore:invalid value:RuntimeWarning")
def test_gradients_that_are_not_finite_stay_in_their_episode(env, dtype):
    """A row gradient, and the gradient of a last state, that are not finite: earlier tokens of the episode get none that
    is finite, other episodes theirs; states are updated in place."""
    torch, S, ctx = env
    for size in ((2, 70, 1, 2, 32, 40), (64, 66, 2, 4, 72, 64), (1, 577, 1, 1, 128, 20)):
        t = size[1]
        d = Delta(env, *size, dtype=dtype, resets=[(0, 5), (0, 20), (0, t - 10)], lengths=[t] * size[0], seed=4)
        clean = d.want_grads()
        d.do[0, 11, 0, 3] = float("nan")
        d.ds[0, 0, 1, 1] = float("inf")
        grads = d.backward(d.forward(True)[2])
        for b in range(1, size[0]):
            for name, x, y in zip(GRADS, grads, clean):
                close(x[b], y[b], name)
        good = np.ones(t, bool)
        good[5:20] = good[t - 10:] = False
        for name, x, y in zip(GRADS[:5], grads, clean):
            close(x[0][torch_mask(x, good)], y[0][good], name)
        close(grads[5][0], clean[5][0], "dstate")
        dv = grads[2][0, :, 0].float().cpu().numpy()
        assert not np.isfinite(dv[5:12, 3]).any() and not np.isfinite(dv[t - 10:, 1]).any()
        close(grads[2][0, 5:20, 0, :3], clean[2][0, 5:20, 0, :3], "columns beside it")
        s, out = d.state.clone(), d.out()[0]
        given = S.DeltaInput(d.q, d.k, d.v, d.g, d.beta, None, s)
        s[0, 0] = float("nan")
        want = O_forward(d, s)
        ctx.pql_delta_forward(d.shape, given, S.Sequence(out), s, None, S.workspace(ctx.delta_workspace_bytes(d.shape, False)))
        close(s, want[1], "state in place")
        close(out[:, 5:], want[0][:, 5:], "out")


def O_forward(d, state):
    from oracle import student_oracle as O
    return O.delta_forward(*d.host, d.scale, None, state.double().cpu().numpy())


# ---- gradient of the distillation by itself ----------------------------------------------------
@pytest.mark.parametrize("rows,vocab", [(5, 50), (40, 900), (5, 2500), (2051, 1500), (3, 70001), (300, 20011)])
@pytest.mark.parametrize("dtype,temp", [("float32", 1.0), ("float32", 0.3), ("bfloat16", 1.5)])
@pytest.mark.parametrize("offset", [40.0, -1000.0, 3e4, LOWEST])
def test_gradient_alone_of_logits_far_from_zero(env, rows, vocab, dtype, temp, offset):
    """Log-sum-exps that 32 bits hold to some 1e-3 or to nothing at all; rows near zero beside them."""
    torch, S, ctx = env
    g = torch.Generator(device="cuda").manual_seed(vocab)
    z = 2 * torch.randn((rows, vocab), generator=g, device="cuda")
    low = torch.finfo(getattr(torch, dtype)).min
    z[:-2] = low if offset == LOWEST else z[:-2] + offset
    z = z.to(getattr(torch, dtype))
    z[-1, 9:] = float("-inf")
    pick = sorted({0, 1, 2, rows // 2, rows - 2, rows - 1})
    host = lambda x: x[pick].double().cpu().numpy()  # noqa: E731
    top = 6
    index = torch.randint(0, vocab, (rows, top), generator=g, device="cuda", dtype=torch.int32)
    index[-1] = torch.arange(top, device="cuda", dtype=torch.int32)
    value = torch.randn((rows, top), generator=g, device="cuda")
    weight = torch.rand((rows,), generator=g, device="cuda") + 0.5
    d, t = S.Logits(z), S.Teacher(index, value)
    loss, lse = (torch.empty((rows,), device="cuda") for _ in range(2))
    ctx.pql_distill_loss(d, t, temp, None, loss, lse, None, S.workspace(ctx.distill_workspace_bytes(d)))
    _, want_lse, want = O_distill(host(z), index[pick].cpu().numpy(), host(value), temp, host(weight))
    close(lse[pick], held(want_lse), "lse")
    grad = torch.full_like(z, 7.0)
    ctx.pql_distill_backward(d, t, temp, lse, weight, S.Logits(grad))
    close(grad[pick], want, "gradient by itself")
    ctx.pql_distill_backward(d, t, temp, lse, weight, d)
    close(z[pick], want, "gradient in place")
    assert torch.equal(z, grad)


def O_distill(*a):
    from oracle import student_oracle as O
    return O.distill(*a)


# ---- one rounding to 16 bits -------------------------------------------------------------------
@pytest.mark.parametrize("t", [1, 40, 600])
def test_outputs_in_16_bits_are_rounded_once(env, t):
    """Outputs a little above the middle of two bfloat16 values, by what lies in the last bits of a state (1 + 2^-9 + 2^-20 and
    2^-9, sum 1 + 2^-8 + 2^-20) and of a product ((1 + 2^-9)^2 = 1 + 2^-8 + 2^-18): both are exact in 32 bits and round up to
    1 + 2^-7; to 1 if any of those bits is lost before."""
    torch, S, ctx = env
    for what in ("state", "product"):
        q, k, v = (torch.zeros((1, t, 1, n), dtype=torch.bfloat16, device="cuda") for n in (2, 2, 1))
        g, beta = torch.zeros((1, t, 1), device="cuda"), torch.zeros((1, t, 1), device="cuda")
        state = torch.zeros((1, 1, 2, 1), device="cuda")
        q[0, 0, 0] = 1.0
        if what == "state":
            state[0, 0, 0, 0], state[0, 0, 1, 0] = 1 + 2.0 ** -9 + 2.0 ** -20, 2.0 ** -9
        else:
            k[0, 0, 0, 0], k[0, 0, 0, 1] = 1.0, 2.0 ** -9
            v[0, 0], beta[0, 0] = 1.0, 1 + 2.0 ** -9
        shape, given = S.delta_shape(q, v, 1.0), S.DeltaInput(q, k, v, g, beta, None, state)
        for call in ("step", "forward"):
            out, last = torch.full_like(v, 7.0), torch.empty_like(state)
            if call == "step":
                ctx.pql_delta_step(shape, given, last, S.Sequence(out))
            else:
                ctx.pql_delta_forward(shape, given, S.Sequence(out), last, None, S.workspace(ctx.delta_workspace_bytes(shape, False)))
            assert float(out[0, 0, 0, 0]) == 1 + 2.0 ** -7, (what, call)


# ---- more rows than one launch takes -------------------------------------------------------------
# Rows repeat with a period that no launch's share is a multiple of, so that the reference is small.  Selections and what is summed
# over tokens repeat bit for bit; sums over a row do not, since where its 16-byte granules lie goes by the row's address.
def periodic(torch, x, n):
    return x.repeat(-(-n // x.shape[0]), *[1] * (x.dim() - 1))[:n].contiguous()


def repeats(x, period):
    return bool((x[period:] == x[:-period]).all())


def close_everywhere(torch, x, want, what):
    """close() for rows that repeat, on the device."""
    want = torch.from_numpy(want).cuda()
    rms, part, err = want.square().mean().sqrt(), len(want) * 40000, 0.0
    for i in range(0, len(x), part):
        got = x[i:i + part].double()
        y = periodic(torch, want, len(got))
        off = (got - y).abs()
        if x.dtype == torch.bfloat16:
            off = (off - torch.exp2(torch.floor(torch.log2(torch.maximum(got.abs(), y.abs()).clamp(min=1e-37))) - 8)).clamp(min=0)
        assert bool((off <= 40 * NORM * torch.maximum(rms, y.abs())).all()), what
        err += float(off.square().sum())
    assert err ** 0.5 <= NORM * float(rms) * x.numel() ** 0.5, what


@pytest.mark.parametrize("rows,vocab,top,dtype", [(2 ** 29 + 3, 2, 1, "bfloat16"), (65539, 1025, 65, "float32"), (65539, 8300, 70, "bfloat16")])
def test_more_rows_than_one_launch_takes(env, rows, vocab, top, dtype):
    torch, S, ctx = env
    period = 97
    rng = np.random.default_rng(top)
    z = torch.from_numpy(2 * rng.standard_normal((period, vocab))).to(getattr(torch, dtype)).cuda()
    host = z.double().cpu().numpy()
    z = periodic(torch, z, rows)
    d = S.Logits(z)
    index, value = torch.full((rows, top), 7, dtype=torch.int32, device="cuda"), torch.full((rows, top), 7.0, device="cuda")
    ctx.pql_top_logits(d, top, index, value, S.workspace(ctx.top_logits_workspace_bytes(d, top)))
    from oracle import student_oracle as O
    want_i, want_v = O.top_logits(host, top)
    assert np.array_equal(index[:period].cpu().numpy(), want_i) and np.array_equal(value[:period].double().cpu().numpy(), want_v)
    assert repeats(index, period) and repeats(value, period)
    value.add_(1.0)
    t = S.Teacher(index, value)
    loss, lse, weight = (torch.full((rows,), 7.0, device="cuda") for _ in range(3))
    grad = torch.full_like(z, 7.0)
    ctx.pql_distill_loss(d, t, 1.0, weight, loss, lse, S.Logits(grad), S.workspace(ctx.distill_workspace_bytes(d)))
    want = O.distill(host, want_i, want_v + 1.0, 1.0, np.full(period, 7.0))
    for name, x, y in zip(("loss", "lse", "grad"), (loss, lse, grad), want):
        close_everywhere(torch, x, y, name)
    ctx.pql_distill_backward(d, t, 1.0, lse, weight, S.Logits(grad.fill_(7)))
    close_everywhere(torch, grad, want[2], "gradient by itself")


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_more_sequences_than_one_launch_takes(env, dtype):
    torch, S, ctx = env
    from oracle import student_oracle as O
    n, period, t, hk, hv, dk, dv = 65539, 37, 3, 1, 2, 4, 3
    d = Delta(env, period, t, hk, hv, dk, dv, dtype=dtype, lengths=[i % (t + 1) for i in range(period)], resets=[(3, 1)], seed=6)
    wide = lambda x: periodic(torch, x, n)  # noqa: E731
    q, k, v, g, beta, do, state, ds = map(wide, (d.q, d.k, d.v, d.g, d.beta, d.do, d.state, d.ds))
    lengths = wide(d.lengths)
    shape, given = S.delta_shape(q, v, d.scale), S.DeltaInput(q, k, v, g, beta, lengths, state)
    out, last = torch.full_like(v, 7.0), torch.full_like(state, 7.0)
    saved = S.workspace(ctx.delta_saved_bytes(shape))
    ctx.pql_delta_forward(shape, given, S.Sequence(out), last, saved, None)
    grads = [torch.full_like(x, 7.0) for x in (q, k, v, g, beta, state)]
    ctx.pql_delta_backward(shape, given, saved, S.Sequence(do), ds, S.DeltaGrad(*grads), S.workspace(ctx.delta_workspace_bytes(shape, True)))
    for name, x, y in zip(("out", "state") + GRADS, [out, last] + grads, [*d.want(), *d.want_grads()]):
        close(x[:period], y, name)
        assert repeats(x, period), name


def test_more_heads_than_one_launch_takes(env):
    """Two sequences in launches of their own, and a key head whose gradient is the sum over 40000 value heads."""
    torch, S, ctx = env
    n, t, period, times, dk, dv = 2, 3, 40, 1000, 4, 3
    d = Delta(env, n, t, 1, period, dk, dv, resets=[(1, 1)], seed=8)
    wide = lambda x, at: x.repeat(*[times if i == at else 1 for i in range(x.dim())])  # noqa: E731
    v, g, beta, do = (wide(x, 2) for x in (d.v, d.g, d.beta, d.do))
    state, ds = wide(d.state, 1), wide(d.ds, 1)
    shape, given = S.delta_shape(d.q, v, d.scale), S.DeltaInput(d.q, d.k, v, g, beta, None, state)
    out, last = torch.full_like(v, 7.0), torch.full_like(state, 7.0)
    saved = S.workspace(ctx.delta_saved_bytes(shape))
    ctx.pql_delta_forward(shape, given, S.Sequence(out), last, saved, None)
    grads = [torch.full_like(x, 7.0) for x in (d.q, d.k, v, g, beta, state)]
    ctx.pql_delta_backward(shape, given, saved, S.Sequence(do), ds, S.DeltaGrad(*grads), S.workspace(ctx.delta_workspace_bytes(shape, True)))
    want = d.want_grads()
    # the sum of 40000 terms in order: the error of one sum of 32-bit numbers grows with sqrt(40000) roundings of 6e-8, 1.2e-5; of terms
    # that repeat, with up to 40000 of them, 2.4e-3
    for name, x, y in zip(("dq", "dk"), grads, want):
        off = np.abs(x.double().cpu().numpy() - times * y)
        assert np.linalg.norm(off) <= 2.4e-3 * np.linalg.norm(times * y), name
    for name, x, y in zip(("out", "state") + GRADS[2:], [out, last] + grads[2:], [*d.want(), *want[2:]]):
        at = 1 if name in ("state", "dstate") else 2
        x = x.transpose(0, at)
        close(x[:period].transpose(0, at), y, name)
        assert repeats(x, period), name


@pytest.mark.parametrize("rows,vocab,top,dtype", [(1, 131072, 32, "float32"), (128, 131072, 9, "float32"), (100, 140009, 1, "bfloat16"),
                                                  (5, 200003, 64, "float32"), (3, 600011, 16, "bfloat16"), (2, 1300021, 64, "float32")])
@pytest.mark.parametrize("levels", [0, 3])
def test_selection_of_long_rows_in_pieces(env, rows, vocab, top, dtype, levels):
    """Lists of pieces joined: distinct logits and a few values that all pieces hold, rows that begin with nothing to select."""
    torch, S, ctx = env
    rng = np.random.default_rng(vocab + levels)
    x = rng.integers(0, levels, (rows, vocab)) if levels else rng.standard_normal((rows, vocab))
    z = torch.from_numpy(x.astype(np.float32)).to(getattr(torch, dtype)).cuda()
    z[0, : vocab // 2] = float("-inf")
    z[-1, vocab // 3:] = float("-inf")
    d = S.Logits(z)
    assert ctx.top_logits_workspace_bytes(d, top) > 0
    index = torch.full((rows, top), 7, dtype=torch.int32, device="cuda")
    value = torch.full((rows, top), 7.0, device="cuda")
    ctx.pql_top_logits(d, top, index, value, S.workspace(ctx.top_logits_workspace_bytes(d, top)))
    from oracle import student_oracle as O
    want_i, want_v = O.top_logits(z.float().cpu().numpy(), top)
    assert np.array_equal(index.cpu().numpy(), want_i)
    assert np.array_equal(value.double().cpu().numpy(), want_v)


@pytest.mark.parametrize("rows,vocab,dtype", [(1, 20011, "float32"), (128, 20000, "float32"), (129, 20000, "float32"), (3, 40009, "bfloat16"), (2, 50021, "float32"),
                                              (1, 300007, "float32"), (1, 300007, "bfloat16")])
def test_loss_of_long_rows_in_pieces_and_whole(env, rows, vocab, dtype):
    """Either side of the rules that cut rows: loss and gradient in one call, each by itself."""
    torch, S, ctx = env
    z, host = logits(torch, rows, vocab, dtype, vocab, True, mask=0.0)
    index, value, weight = lists(rows, vocab, 40, vocab + 1)
    z[:], host = torch.nan_to_num(z, neginf=-1.0), np.nan_to_num(host, neginf=-1.0)
    d, t, w = S.Logits(z), S.Teacher(torch.from_numpy(index).cuda(), torch.from_numpy(value).cuda()), torch.from_numpy(weight).cuda()
    loss, lse = (torch.full((rows,), 7.0, device="cuda") for _ in range(2))
    grad = torch.full((rows, vocab), 7.0, dtype=z.dtype, device="cuda")
    ws = S.workspace(ctx.distill_workspace_bytes(d))
    want = O_distill(host, index, value, 1.5, weight)
    ctx.pql_distill_loss(d, t, 1.5, w, loss, lse, S.Logits(grad), ws)
    for name, x, y in zip(("loss", "lse", "grad"), (loss, lse, grad), want):
        close(x, y, name)
    ctx.pql_distill_loss(d, t, 1.5, w, loss.fill_(7), lse.fill_(7), None, ws)
    close(loss, want[0], "loss alone")
    ctx.pql_distill_loss(d, t, 1.5, None, loss, lse, None, ws)
    ctx.pql_distill_backward(d, t, 1.5, lse, w, S.Logits(grad.fill_(7)))
    close(grad, want[2], "gradient by itself")
