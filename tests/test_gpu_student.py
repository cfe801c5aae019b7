"""The student's operators on the GPU against the double-precision reference.

Tolerances, from the arithmetic: every product is accumulated in 32 bits (unit roundoff 6e-8) over at most 192
terms and the longest chain from an input to an output has about six products, so the 2-norm of an error is below
sqrt(192) * 6 * 6e-8 * (a condition of two) = 1e-5 of the result's.  An output in bfloat16 is rounded once, by at
most half the spacing of its values: what it is off beyond that obeys the same bound.  Single elements may be off by
40 times the bound of the norm, relative to the larger of the element and the root mean square.  The distillation's sums are shorter: the same bounds hold.  Selected
logits are compared bit for bit."""
import numpy as np
import pytest

from oracle import student_oracle as O

pytestmark = pytest.mark.gpu
NORM = 1e-5


@pytest.fixture(scope="module")
def env():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible: the gpu-marked tests need a real MI355X")
    from paper_2307_12983_amd import student as S
    return torch, S, S.StudentContext()


def close(got, want, what):
    bf16 = str(got.dtype) == "torch.bfloat16"
    got = got.detach().double().cpu().numpy()
    want = np.asarray(want, np.float64)
    assert got.shape == want.shape, what
    fine = np.isfinite(want)
    assert np.array_equal(fine, np.isfinite(got)), what + ": not finite where it should be, or the reverse"
    assert np.array_equal(got[~fine], want[~fine]), what
    got, want = got[fine], want[fine]
    norm = np.linalg.norm(want)
    off = np.abs(got - want)
    if bf16:                                            # 8 significant bits: half a spacing is 2^(exponent - 8)
        size = np.maximum(np.abs(got), np.abs(want))
        off = np.maximum(0.0, off - np.exp2(np.floor(np.log2(np.maximum(size, 1e-37))) - 8))
    err = np.linalg.norm(off)
    assert err <= NORM * norm, "%s: error %.3g of the norm" % (what, err / norm if norm else np.inf)
    if norm:
        worst = np.max(off / np.maximum(norm / np.sqrt(want.size), np.abs(want)))
        assert worst <= 40 * NORM, "%s: an element off by %.3g" % (what, worst)


class Delta:
    """One set of inputs in a layout, and the calls on it."""

    def __init__(self, env, n, t, hk, hv, dk, dv, dtype="float32", layout="dense", lengths=None, resets=(), keys="random",
                 state=True, seed=0, beta_top=1.0):
        torch, S, ctx = self.env = env
        rng = np.random.default_rng(seed)
        dt = getattr(torch, dtype)
        unit = lambda x: x / np.linalg.norm(x, axis=-1, keepdims=True)  # noqa: E731
        k = rng.standard_normal((n, t, hk, dk))
        if keys == "equal":
            k = np.broadcast_to(k[:, :1], k.shape)
        k, q = unit(k), unit(rng.standard_normal((n, t, hk, dk)))
        v = rng.standard_normal((n, t, hv, dv))
        g = -0.5 * rng.random((n, t, hv)) ** 2
        for b, i in resets:
            if b < n and i < t:
                g[b, i] = -np.inf
        beta = beta_top * rng.random((n, t, hv))
        dev = lambda x, d=torch.float32: torch.tensor(np.ascontiguousarray(x), dtype=torch.float64).to(d).cuda()  # noqa: E731
        q, k, v = dev(q, dt), dev(k, dt), dev(v, dt)
        do = dev(rng.standard_normal((n, t, hv, dv)), dt)
        if layout == "packed":
            rows = torch.cat([q.flatten(2), k.flatten(2), v.flatten(2)], -1)
            q, k, v = rows.split([hk * dk, hk * dk, hv * dv], -1)
            q, k, v = q.unflatten(-1, (hk, dk)), k.unflatten(-1, (hk, dk)), v.unflatten(-1, (hv, dv))
        elif layout == "heads_first":
            q, k, v, do = (x.transpose(1, 2).contiguous().transpose(1, 2) for x in (q, k, v, do))
        elif layout == "offset":                       # rows that start on no 16-byte boundary
            def shift(x):
                big = torch.zeros((*x.shape[:-1], x.shape[-1] + 3), dtype=x.dtype, device="cuda")
                big[..., 1:1 + x.shape[-1]] = x
                return big[..., 1:1 + x.shape[-1]]
            q, k, v, do = map(shift, (q, k, v, do))
        elif layout == "broadcast":                    # one key sequence and one gradient row for every sequence
            k, do = k[:1].expand(n, -1, -1, -1), do[:, :1].expand(-1, t, -1, -1)
        self.q, self.k, self.v, self.do = q, k, v, do
        self.g, self.beta = dev(g), dev(beta)
        if layout == "heads_first":
            self.g, self.beta = (x.transpose(1, 2).contiguous().transpose(1, 2) for x in (self.g, self.beta))
        self.state = dev(0.5 * rng.standard_normal((n, hv, dk, dv))) if state else None
        self.ds = dev(rng.standard_normal((n, hv, dk, dv))) if state else None
        self.lengths = None if lengths is None else torch.tensor(lengths, dtype=torch.int32).cuda()
        self.lens = lengths
        self.scale = float(np.float32(dk ** -0.5))
        self.shape = S.delta_shape(q, v, self.scale)
        self.given = S.DeltaInput(q, k, v, self.g, self.beta, self.lengths, self.state)
        self.host = [x.double().cpu().numpy() for x in (q, k, v, self.g, self.beta)]
        self.host_state = None if self.state is None else self.state.double().cpu().numpy()

    def poison(self):
        """NaN behind every length: nothing there may be read."""
        torch = self.env[0]
        for b, length in enumerate(self.lens):
            for x in (self.q, self.k, self.v, self.g, self.beta, self.do):
                x[b, max(0, length):] = float("nan")
        torch.cuda.synchronize()
        return self

    def out(self):
        torch = self.env[0]
        n, t, hv, dv = self.v.shape
        return torch.full((n, t, hv, dv), 7.0, dtype=self.v.dtype, device="cuda"), torch.full((n, hv, self.q.shape[3], dv), 7.0, device="cuda")

    def step(self):
        _, S, ctx = self.env
        out, state = self.out()
        ctx.pql_delta_step(self.shape, self.given, state, S.Sequence(out))
        return out, state

    def forward(self, save=False):
        _, S, ctx = self.env
        out, state = self.out()
        saved = S.workspace(ctx.delta_saved_bytes(self.shape)) if save else None
        ws = S.workspace(ctx.delta_workspace_bytes(self.shape, False))
        ctx.pql_delta_forward(self.shape, self.given, S.Sequence(out), state, saved, ws)
        return (out, state, saved) if save else (out, state)

    def backward(self, saved):
        torch, S, ctx = self.env
        full = lambda x: torch.full(x.shape, 7.0, dtype=x.dtype, device="cuda")  # noqa: E731
        grads = [full(x) for x in (self.q, self.k, self.v, self.g, self.beta)] + [None if self.state is None else full(self.state)]
        ws = S.workspace(ctx.delta_workspace_bytes(self.shape, True))
        ctx.pql_delta_backward(self.shape, self.given, saved, S.Sequence(self.do), self.ds, S.DeltaGrad(*grads), ws)
        return grads

    def want(self):
        return O.delta_forward(*self.host, self.scale, self.lens, self.host_state)

    def want_grads(self):
        ds = None if self.ds is None else self.ds.double().cpu().numpy()
        return O.delta_backward(*self.host, self.scale, np.nan_to_num(self.do.double().cpu().numpy()), ds, self.lens, self.host_state)


SHAPES = [(1, 1, 1, 1, 1, 1), (2, 2, 1, 1, 3, 5), (2, 64, 1, 1, 64, 32), (2, 65, 2, 4, 16, 17), (1, 130, 1, 2, 128, 128),
          (2, 200, 3, 3, 72, 100), (1, 190, 1, 1, 128, 256), (3, 63, 2, 2, 7, 40), (2, 129, 2, 6, 33, 64), (1, 70, 1, 1, 64, 65)]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("size", SHAPES)
def test_forms_of_the_delta_rule(env, size, dtype):
    d = Delta(env, *size, dtype=dtype, resets=[(0, 0), (0, 40), (1, 63), (1, 64), (1, 65)], seed=size[1])
    out, state = d.want()
    for name, got in (("step", d.step()), ("forward", d.forward()), ("forward, kept", d.forward(True)[:2])):
        close(got[0], out, name + " out")
        close(got[1], state, name + " state")


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("size", SHAPES)
def test_gradients_of_the_delta_rule(env, size, dtype):
    d = Delta(env, *size, dtype=dtype, resets=[(0, 0), (0, 40), (1, 63), (1, 64), (1, 65)], seed=size[1])
    grads = d.backward(d.forward(True)[2])
    for name, got, want in zip(("dq", "dk", "dv", "dg", "dbeta", "dstate"), grads, d.want_grads()):
        close(got, want, name)


@pytest.mark.parametrize("layout", ["packed", "heads_first", "offset", "broadcast"])
@pytest.mark.parametrize("dtype,size", [("float32", (2, 70, 2, 4, 32, 48)), ("bfloat16", (2, 70, 2, 2, 64, 40))])
def test_layouts(env, layout, dtype, size):
    d = Delta(env, *size, dtype=dtype, layout=layout, resets=[(1, 20)], seed=5)
    out, state = d.want()
    for got in (d.step(), d.forward()):
        close(got[0], out, layout + " out")
        close(got[1], state, layout + " state")
    for name, got, want in zip(("dq", "dk", "dv", "dg", "dbeta", "dstate"), d.backward(d.forward(True)[2]), d.want_grads()):
        close(got, want, layout + " " + name)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("state", [True, False])
def test_lengths(env, dtype, state):
    """Empty, one-token, chunk-ending and over-long lengths; nothing behind them is read, zeros are written there."""
    lens = [0, 1, 64, 63, 65, 128, 140, 200, -3]
    d = Delta(env, len(lens), 140, 1, 2, 16, 24, dtype=dtype, lengths=lens, resets=[(4, 10), (5, 127)], state=state, seed=9).poison()
    d.host = [np.nan_to_num(x, nan=0.0, posinf=np.inf, neginf=-np.inf) for x in d.host]
    out, s = d.want()
    grads_want = d.want_grads()
    for got in (d.step(), d.forward()):
        close(got[0], out, "out")
        close(got[1], s, "state")
    for name, got, want in zip(("dq", "dk", "dv", "dg", "dbeta", "dstate"), d.backward(d.forward(True)[2]), grads_want):
        if got is not None:
            close(got, want, name)


def test_equal_keys_and_strong_writes(env):
    """Keys that are all the same make (I + N diag(beta)) as ill-suited to a series as it gets; beta up to 2."""
    for dtype in ("float32", "bfloat16"):
        d = Delta(env, 2, 128, 1, 1, 64, 32, dtype=dtype, keys="equal", seed=2)
        got = d.forward(True)
        out, state = d.want()
        close(got[0], out, "out")
        close(got[1], state, "state")
        for name, x, y in zip(("dq", "dk", "dv", "dg", "dbeta", "dstate"), d.backward(got[2]), d.want_grads()):
            close(x, y, name)
    d = Delta(env, 1, 100, 1, 1, 64, 32, beta_top=2.0, seed=3)
    got, (out, state) = d.forward(), d.want()
    close(got[0], out, "out")
    close(got[1], state, "state")


def test_a_reset_forgets_states_that_are_not_finite(env):
    d = Delta(env, 1, 70, 1, 1, 16, 16, resets=[(0, 0), (0, 66)], seed=4)
    d.state.fill_(float("inf"))
    d.host_state = np.zeros_like(d.host_state)
    out, state = d.want()
    for name, got in (("step", d.step()), ("forward", d.forward())):
        close(got[0], out, name + " out")
        close(got[1], state, name + " state")
    for name, x, y in zip(("dq", "dk", "dv", "dg", "dbeta", "dstate"), d.backward(d.forward(True)[2]), d.want_grads()):
        close(x, y, name)


def test_state_in_place_no_state_out_and_zero_steps(env):
    torch, S, ctx = env
    d = Delta(env, 3, 5, 1, 2, 32, 20, lengths=[0, 5, 2], seed=6)
    out, state = d.want()
    for call in ("step", "forward"):
        s = d.state.clone()
        given = S.DeltaInput(d.q, d.k, d.v, d.g, d.beta, d.lengths, s)
        o, _ = d.out()
        ws = S.workspace(ctx.delta_workspace_bytes(d.shape, False))
        if call == "step":
            ctx.pql_delta_step(d.shape, given, s, S.Sequence(o))
        else:
            ctx.pql_delta_forward(d.shape, given, S.Sequence(o), s, None, ws)
        close(o, out, call + " out")
        close(s, state, call + " state")
    o, _ = d.out()
    ctx.pql_delta_forward(d.shape, d.given, S.Sequence(o), None, None, ws)
    close(o, out, "out without a state")
    e = Delta(env, 2, 0, 1, 1, 8, 8, seed=1)
    for got in (e.step(), e.forward()):
        assert torch.equal(got[1], e.state)
    assert torch.equal(e.backward(S.workspace(256))[5], e.ds)


def test_calls_repeat_bit_for_bit_on_another_stream_and_in_a_graph(env):
    torch, S, ctx = env
    d = Delta(env, 2, 130, 1, 2, 64, 64, dtype="bfloat16", seed=8)
    first = d.forward(True)
    grads = d.backward(first[2])
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        again = d.forward(True)
        more = d.backward(again[2])
    stream.synchronize()
    for x, y in zip(list(first[:2]) + grads, list(again[:2]) + more):
        assert torch.equal(x, y)
    o, s = d.out()
    o_d, saved = S.Sequence(o), S.workspace(ctx.delta_saved_bytes(d.shape))
    ws = S.workspace(ctx.delta_workspace_bytes(d.shape, True))
    g = [torch.zeros_like(x) for x in (d.q, d.k, d.v, d.g, d.beta, d.state)]
    g_d, do = S.DeltaGrad(*g), S.Sequence(d.do)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.pql_delta_forward(d.shape, d.given, o_d, s, saved, ws)
        ctx.pql_delta_backward(d.shape, d.given, saved, do, d.ds, g_d, ws)
    for _ in range(3):
        for x in [o, s] + g:
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(list(first[:2]) + grads, [o, s] + g):
            assert torch.equal(x, y)


# ---- rows of logits ---------------------------------------------------------------------------
ROWS = [(1, 1, 1), (7, 2, 2), (33, 51, 8), (5, 64, 64), (9, 65, 3), (6, 130, 100), (4, 1000, 256), (3, 1024, 7), (6, 1025, 32),
        (3, 1500, 256), (520, 1501, 4), (2, 70001, 100), (515, 4099, 256), (1, 20000, 1)]


def logits(torch, rows, vocab, dtype, seed, offset, mask=0.15, levels=0):
    rng = np.random.default_rng(seed)
    z = 2 * rng.standard_normal((rows, vocab))
    if levels:
        z = rng.integers(0, levels, (rows, vocab)).astype(np.float64)
    z[rng.random((rows, vocab)) < mask] = -np.inf
    if rows > 2:
        z[1] = -np.inf
    dt = getattr(torch, dtype)
    if offset:
        big = torch.zeros((rows, vocab + 5), dtype=dt, device="cuda")
        t = big[:, 3:3 + vocab]
        t.copy_(torch.from_numpy(z))
    else:
        t = torch.from_numpy(z).to(dt).cuda()
    return t, t.double().cpu().numpy()


@pytest.mark.parametrize("offset", [False, True])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows,vocab,top", ROWS)
def test_top_logits(env, rows, vocab, top, dtype, offset):
    torch, S, ctx = env
    for levels in (0, 3):                               # few levels: ties by the thousand
        z, host = logits(torch, rows, vocab, dtype, vocab + levels, offset, levels=levels)
        if rows > 3 and vocab > 4:
            z[3, :3] = float("nan")
            host[3, :3] = np.nan
        d = S.Logits(z)
        index = torch.full((rows, top), 7, dtype=torch.int32, device="cuda")
        value = torch.full((rows, top), 7.0, device="cuda")
        ctx.pql_top_logits(d, top, index, value, S.workspace(ctx.top_logits_workspace_bytes(d, top)))
        want_i, want_v = O.top_logits(host, top)
        assert np.array_equal(index.cpu().numpy(), want_i), "indices, %d levels" % levels
        assert np.array_equal(value.double().cpu().numpy(), want_v), "values, %d levels" % levels


def test_top_logits_equal_negative_and_zero_values(env):
    torch, S, ctx = env
    for vocab in (40, 3000):
        z = torch.full((3, vocab), -2.5, device="cuda")
        z[1, ::2] = 0.0
        z[1, 1::2] = -0.0                               # equal to +0
        z[2] = torch.finfo(torch.float32).min
        d = S.Logits(z)
        index, value = torch.empty((3, 9), dtype=torch.int32, device="cuda"), torch.empty((3, 9), device="cuda")
        ctx.pql_top_logits(d, 9, index, value, S.workspace(ctx.top_logits_workspace_bytes(d, 9)))
        assert torch.equal(index.cpu(), torch.arange(9, dtype=torch.int32).expand(3, 9))
        assert torch.equal(value, z[:, :9])


def lists(rows, vocab, top, seed):
    rng = np.random.default_rng(seed)
    index = np.argsort(rng.random((rows, vocab)), axis=1)[:, :top].astype(np.int32) if vocab < 5000 else \
        rng.integers(0, vocab, (rows, top)).astype(np.int32)
    value = (2 * rng.standard_normal((rows, top))).astype(np.float32)
    if top > 2:
        index[0, top // 2] = -1                         # no entry, in the middle of a list
        index[-1, 1] = index[-1, 0]                     # an answer listed twice
        value[-1, 2] = -np.inf
    if rows > 4:
        index[2] = -1                                   # an empty list
        index[4, -1] = vocab                            # outside
    weight = (0.5 + rng.random(rows)).astype(np.float32)
    if rows > 5:
        weight[5] = 0.0
    return index, value, weight


@pytest.mark.parametrize("offset", [False, True])
@pytest.mark.parametrize("dtype,temp", [("float32", 1.0), ("float32", 3.0), ("bfloat16", 0.5)])
@pytest.mark.parametrize("rows,vocab,top", ROWS)
def test_distillation(env, rows, vocab, top, dtype, temp, offset):
    torch, S, ctx = env
    z, host = logits(torch, rows, vocab, dtype, vocab, offset, mask=0.0)
    index, value, weight = lists(rows, vocab, top, vocab + 1)
    if vocab > 10:                                      # masked answers that no list holds
        free = np.ones((rows, vocab), bool)
        for n in range(rows):
            free[n, index[n][(index[n] >= 0) & (index[n] < vocab)]] = False
        free &= np.random.default_rng(5).random((rows, vocab)) < 0.1
        host = np.where(free, -np.inf, np.nan_to_num(host, neginf=-1.0))
        z.copy_(torch.from_numpy(host))
        host = z.double().cpu().numpy()
    else:
        host = np.nan_to_num(host, neginf=-1.0)
        z.copy_(torch.from_numpy(host))
        host = z.double().cpu().numpy()
    if rows > 5:
        z[5], z[2] = float("nan"), float("nan")         # rows that are not read
    d = S.Logits(z)
    t = S.Teacher(torch.from_numpy(index).cuda(), torch.from_numpy(value).cuda())
    w = torch.from_numpy(weight).cuda()
    loss, lse = (torch.full((rows,), 7.0, device="cuda") for _ in range(2))
    grad = torch.full((rows, vocab), 7.0, dtype=z.dtype, device="cuda")
    ws = S.workspace(ctx.distill_workspace_bytes(d))
    want = O.distill(host, index, value, temp, weight)
    plain = O.distill(host, index, value, temp)
    ctx.pql_distill_loss(d, t, temp, w, loss, lse, S.Logits(grad), ws)
    for name, x, y in zip(("loss", "lse", "grad"), (loss, lse, grad), want):
        close(x, y, name)
    ctx.pql_distill_loss(d, t, temp, w, loss.fill_(7), lse.fill_(7), None, ws)
    close(loss, want[0], "loss alone")
    # the two calls: the loss without weights, then the gradient for given row gradients
    if rows > 5:
        z[5] = torch.from_numpy(host[5]).to(z.dtype).cuda()
    ctx.pql_distill_loss(d, t, temp, None, loss.fill_(7), lse.fill_(7), None, ws)
    close(loss, plain[0], "loss without weights")
    close(lse, plain[1], "lse without weights")
    if rows > 5:
        z[5] = float("nan")
    ctx.pql_distill_backward(d, t, temp, lse, w, S.Logits(grad.fill_(7)))
    close(grad, want[2], "gradient by itself")
    ctx.pql_distill_backward(d, t, temp, lse, w, d)     # in the logits' place
    close(z, want[2], "gradient in place")


@pytest.mark.parametrize("rows,vocab", [(6, 60), (6, 3000), (600, 2000)])
def test_distillation_in_place_and_of_masked_answers(env, rows, vocab):
    torch, S, ctx = env
    z, host = logits(torch, rows, vocab, "float32", 1, False, mask=0.5)     # listed answers among the masked; row 1 empty
    index, value, weight = lists(rows, vocab, 6, 3)
    weight[1] = 1.0
    t = S.Teacher(torch.from_numpy(index).cuda(), torch.from_numpy(value).cuda())
    loss, lse = (torch.empty((rows,), device="cuda") for _ in range(2))
    d = S.Logits(z)
    ctx.pql_distill_loss(d, t, 2.0, torch.from_numpy(weight).cuda(), loss, lse, d, S.workspace(ctx.distill_workspace_bytes(d)))
    want = O.distill(host, index, value, 2.0, weight)
    assert np.isinf(want[0]).any() and want[1][1] == -np.inf
    for name, x, y in zip(("loss", "lse", "grad"), (loss, lse, z), want):
        close(x, y, name)


def test_distillation_with_the_lowest_values_as_masks(env):
    torch, S, ctx = env
    for dtype in ("float32", "bfloat16"):
        for vocab in (50, 2500):
            low = torch.finfo(getattr(torch, dtype)).min
            z, host = logits(torch, 4, vocab, dtype, 7, False, mask=0.0)
            z[0, 10:] = low
            z[1] = low                                  # all of them: a uniform row
            host = z.double().cpu().numpy()
            index = np.arange(4, dtype=np.int32)[None].repeat(4, 0)
            value = np.random.default_rng(1).standard_normal((4, 4)).astype(np.float32)
            t = S.Teacher(torch.from_numpy(index).cuda(), torch.from_numpy(value).cuda())
            loss, lse = (torch.empty((4,), device="cuda") for _ in range(2))
            grad, d = torch.empty_like(z), S.Logits(z)
            ctx.pql_distill_loss(d, t, 1.0, None, loss, lse, S.Logits(grad), S.workspace(ctx.distill_workspace_bytes(d)))
            for name, x, y in zip(("loss", "lse", "grad"), (loss, lse, grad), O.distill(host, index, value, 1.0)):
                close(x, y, name)


def test_kernels_are_timed_under_their_names(env):
    torch, S, ctx = env
    d = Delta(env, 1, 70, 1, 2, 16, 16, seed=1)
    ctx.pql_profile_begin(32)
    d.step()
    d.backward(d.forward(True)[2])
    names = {k["name"]: k for k in ctx.pql_profile_end()}
    assert set(names) == {"delta_step_kernel", "delta_prepare_kernel", "delta_scan_kernel", "delta_back_scan_kernel",
                          "delta_back_kernel", "delta_group_kernel"}
    assert all(k["launches"] == 1 and k["total_ms"] > 0 for k in names.values())


SHORT = [(3, 32, 2, 4, 64, 64), (2, 31, 1, 2, 128, 96), (5, 17, 1, 1, 72, 36), (2, 16, 3, 3, 20, 130)]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("size", SHORT)
def test_windows_of_at_most_32_tokens(env, size, dtype):
    n, t = size[:2]
    lens = [t, 0, 1, t - 1, 9][:n]
    d = Delta(env, *size, dtype=dtype, lengths=lens, resets=[(0, 0), (0, 7), (0, 8), (0, t - 1), (3, 3)], seed=t)
    out, state = d.want()
    want = d.want_grads()
    got = d.forward(True)
    close(got[0], out, "out")
    close(got[1], state, "state")
    for name, x, y in zip(("dq", "dk", "dv", "dg", "dbeta", "dstate"), d.backward(got[2]), want):
        close(x, y, name)


@pytest.mark.parametrize("dtype,size", [("float32", (512, 3, 1, 2, 16, 8)), ("bfloat16", (86, 130, 2, 6, 8, 12)), ("float32", (43, 129, 4, 8, 70, 8))])
def test_gradients_of_shared_heads_in_large_calls(env, dtype, size):
    """Enough chunks for one workgroup to take all value heads of a key head."""
    n, t = size[:2]
    rng = np.random.default_rng(1)
    lens = rng.integers(0, t + 1, n).tolist()
    d = Delta(env, *size, dtype=dtype, lengths=lens, resets=[(b, int(rng.integers(0, t))) for b in range(0, n, 3)], seed=7)
    for name, got, want in zip(("dq", "dk", "dv", "dg", "dbeta", "dstate"), d.backward(d.forward(True)[2]), d.want_grads()):
        close(got, want, name)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("vocab", [4100, 9001, 20011, 40003, 70001, 140009])
def test_rows_of_every_length_class(env, vocab, dtype):
    """One workgroup per row, from rows that a few registers hold to rows that none do: loss, gradient, selection."""
    torch, S, ctx = env
    rows, top = 530, 9
    g = torch.Generator(device="cuda").manual_seed(vocab)
    z = (2 * torch.randn((rows, vocab + 1), generator=g, device="cuda")).to(getattr(torch, dtype))[:, 1:]
    z[3], z[4, 5:] = float("-inf"), float("-inf")
    pick = [0, 1, 3, 4, rows - 1]
    index = torch.randint(0, vocab, (rows, top), generator=g, device="cuda", dtype=torch.int32)
    index[4] = torch.arange(top, device="cuda", dtype=torch.int32) % 5
    value = torch.randn((rows, top), generator=g, device="cuda")
    d = S.Logits(z)
    loss, lse = (torch.full((rows,), 7.0, device="cuda") for _ in range(2))
    grad = torch.full((rows, vocab), 7.0, dtype=z.dtype, device="cuda")
    ctx.pql_distill_loss(d, S.Teacher(index, value), 1.5, None, loss, lse, S.Logits(grad), S.workspace(ctx.distill_workspace_bytes(d)))
    want = O.distill(z[pick].double().cpu().numpy(), index[pick].cpu().numpy(), value[pick].cpu().numpy(), 1.5)
    for name, x, y in zip(("loss", "lse", "grad"), (loss, lse, grad), want):
        close(x[pick], y, name)
    i, v = torch.full((rows, top), 7, dtype=torch.int32, device="cuda"), torch.full((rows, top), 7.0, device="cuda")
    ctx.pql_top_logits(d, top, i, v, S.workspace(ctx.top_logits_workspace_bytes(d, top)))
    want_i, want_v = O.top_logits(z[pick].double().cpu().numpy(), top)
    assert np.array_equal(i[pick].cpu().numpy(), want_i) and np.array_equal(v[pick].double().cpu().numpy(), want_v)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("vocab,top,levels", [(1025, 9, 0), (1500, 64, 0), (2053, 65, 0), (4095, 30, 0), (4096, 3, 40), (8000, 64, 3), (2600, 200, 5)])
def test_many_rows_of_medium_length(env, vocab, top, levels, dtype):
    """Enough rows for one wavefront each: selection with and without ties, loss, gradient in one call and by itself, in place."""
    torch, S, ctx = env
    rows, temp = 2051, 1.25
    g = torch.Generator(device="cuda").manual_seed(vocab)
    z = 2 * torch.randn((rows, vocab + 3), generator=g, device="cuda")
    if levels:
        z = torch.randint(0, levels, z.shape, generator=g, device="cuda").float()
    z = z.to(getattr(torch, dtype))[:, 2:2 + vocab]
    z[1], z[2, 7:], z[3, ::2] = float("-inf"), float("-inf"), float("-inf")
    z[5, 100:110] = float("nan")
    pick = [0, 1, 2, 3, 4, 5, 6, 7, rows - 2, rows - 1]
    host = lambda t: t[pick].double().cpu().numpy()  # noqa: E731
    i, v = torch.full((rows, top), 7, dtype=torch.int32, device="cuda"), torch.full((rows, top), 7.0, device="cuda")
    d = S.Logits(z)
    ctx.pql_top_logits(d, top, i, v, S.workspace(ctx.top_logits_workspace_bytes(d, top)))
    want_i, want_v = O.top_logits(host(z), top)
    assert np.array_equal(i[pick].cpu().numpy(), want_i) and np.array_equal(host(v), want_v)
    z[5] = z[6]
    i[0, top // 2:] = -1                                # a short list, an empty one, an answer twice, a row of no weight
    i[4] = -1
    i[7, -1] = i[7, 0]
    weight = torch.rand((rows,), generator=g, device="cuda") + 0.5
    weight[6] = 0.0
    y = torch.where(torch.isfinite(v), v, 0.0) + torch.randn(v.shape, generator=g, device="cuda")
    t = S.Teacher(i, y)
    loss, lse = (torch.full((rows,), 7.0, device="cuda") for _ in range(2))
    grad = torch.full((rows, vocab), 7.0, dtype=z.dtype, device="cuda")
    ws = S.workspace(ctx.distill_workspace_bytes(d))
    want = O.distill(host(z), i[pick].cpu().numpy(), host(y), temp, host(weight))
    ctx.pql_distill_loss(d, t, temp, weight, loss, lse, S.Logits(grad), ws)
    for name, x, w in zip(("loss", "lse", "grad"), (loss, lse, grad), want):
        close(x[pick], w, name)
    ctx.pql_distill_loss(d, t, temp, None, loss.fill_(7), lse.fill_(7), None, ws)
    plain = O.distill(host(z), i[pick].cpu().numpy(), host(y), temp)
    close(loss[pick], plain[0], "loss alone")
    close(lse[pick], plain[1], "lse alone")
    ctx.pql_distill_backward(d, t, temp, lse, weight, S.Logits(grad.fill_(7)))
    close(grad[pick], want[2], "gradient by itself")
    ctx.pql_distill_backward(d, t, temp, lse, weight, d)
    close(z[pick], want[2], "gradient in place")


# few sequences over 512 tokens go by longer chunks than all others
LONG = [(2, 520, 1, 2, 64, 64), (1, 577, 2, 2, 128, 96), (1, 515, 1, 3, 72, 36), (2, 600, 1, 1, 20, 130), (1, 641, 1, 1, 33, 65),
        (7, 600, 4, 8, 16, 8), (7, 600, 4, 8, 70, 8), (64, 513, 2, 2, 16, 64), (64, 513, 2, 2, 70, 64)]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("size", LONG)
def test_few_long_sequences(env, size, dtype):
    n, t = size[:2]
    lens = ([t, 0, 1, t - 1, 65, 64, 63] + [(97 * i) % (t + 1) for i in range(n)])[:n]
    resets = [(0, 0), (0, 63), (0, 64), (0, 65), (0, t - 1), (3 % n, 300)]
    d = Delta(env, *size, dtype=dtype, lengths=lens, resets=resets, seed=t)
    out, state = d.want()
    kept = d.forward(True)
    for name, got in (("forward", d.forward()), ("forward, kept", kept[:2])):
        close(got[0], out, name + " out")
        close(got[1], state, name + " state")
    for name, x, y in zip(("dq", "dk", "dv", "dg", "dbeta", "dstate"), d.backward(kept[2]), d.want_grads()):
        close(x, y, name)


@pytest.mark.parametrize("top", [13, 17, 24, 49])
@pytest.mark.parametrize("vocab", [64, 100, 250, 500, 1000])
def test_short_rows_and_long_lists(env, vocab, top):
    """Either side of the list lengths at which short rows change from rounds to bits, with many equal logits."""
    torch, S, ctx = env
    rng = np.random.default_rng(vocab + top)
    for dtype in (torch.float32, torch.bfloat16):
        z = torch.from_numpy(rng.integers(-20, 20, (37, vocab)).astype(np.float32)).to(dtype).cuda()
        z[3] = -float("inf")
        z[5, 10:] = float("nan")
        index = torch.empty(37, top, dtype=torch.int32, device="cuda")
        value = torch.empty(37, top, device="cuda")
        ctx.pql_top_logits(S.Logits(z), top, index, value, None)
        want_i, want_v = O.top_logits(z.float().cpu().numpy(), top)
        assert np.array_equal(index.cpu().numpy(), want_i)
        assert np.array_equal(value.cpu().numpy(), want_v)


@pytest.mark.parametrize("rows,vocab,top", [(1, 131072, 256), (3, 70001, 64), (2, 40000, 1), (17, 32768, 100), (255, 33000, 5), (256, 33000, 5)])
@pytest.mark.parametrize("levels", [3, 0])
def test_pieces_of_long_rows(env, rows, vocab, top, levels):
    """Lists of pieces joined: distinct logits, and a few values that all pieces hold."""
    torch, S, ctx = env
    rng = np.random.default_rng(rows + vocab)
    x = rng.integers(0, levels, (rows, vocab)) if levels else rng.standard_normal((rows, vocab))
    z = torch.from_numpy(x.astype(np.float32)).cuda()
    z[0, : vocab // 2] = -float("inf")
    d = S.Logits(z)
    index = torch.empty(rows, top, dtype=torch.int32, device="cuda")
    value = torch.empty(rows, top, device="cuda")
    ctx.pql_top_logits(d, top, index, value, S.workspace(ctx.top_logits_workspace_bytes(d, top)))
    want_i, want_v = O.top_logits(z.cpu().numpy(), top)
    assert np.array_equal(index.cpu().numpy(), want_i)
    assert np.array_equal(value.cpu().numpy(), want_v)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("size", [(1, 40, 1, 2, 64, 64), (1, 40, 1, 1, 100, 24), (128, 40, 2, 2, 64, 64), (128, 40, 2, 2, 72, 64),
                                  (1, 520, 1, 1, 64, 16), (1, 520, 1, 1, 128, 40), (64, 513, 2, 2, 16, 64)])
def test_tokens_far_apart(env, size, dtype):
    """Tokens 2^21 elements and more from one to the next: a chunk is out of reach of 32-bit offsets."""
    torch, S, ctx = env
    d = Delta(env, *size, dtype=dtype, resets=[(0, 0), (0, 33)], seed=3)

    def far(x):
        n, t, h, dim = x.shape
        big = torch.empty((t - 1) * 2 ** 21 + n * h * dim, dtype=x.dtype, device="cuda")
        y = big.as_strided(x.shape, (h * dim, 2 ** 21, dim, 1))
        y.copy_(x)
        return y
    d.v, d.do, d.k = far(d.v), far(d.do), far(d.k)
    d.given = S.DeltaInput(d.q, d.k, d.v, d.g, d.beta, d.lengths, d.state)
    out, state = d.want()
    kept = d.forward(True)
    for name, got in (("step", d.step()), ("forward", d.forward()), ("forward, kept", kept[:2])):
        close(got[0], out, name + " out")
        close(got[1], state, name + " state")
    for name, x, y in zip(("dq", "dk", "dv", "dg", "dbeta", "dstate"), d.backward(kept[2]), d.want_grads()):
        close(x, y, name)
