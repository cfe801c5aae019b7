"""The example that runs the operators of a block with the student's memory and loss.

Tolerances: its longest chain is about ten operators in fp32, each within 1e-5 of the exact result (2-norm, the bounds their own
tests derive) and each with a condition of about two to the next; norms of sums of terms of one size keep that.  Logits and
states by steps and as one window are therefore within 2 * 10 * 2 * 1e-5 = 4e-4 of each other, and gradients, whose chain is
twice as long, within 8e-4 of those in double precision."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def example():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible: the gpu-marked tests need a real MI355X")
    import block_student
    return torch, block_student


def test_a_student_of_a_block_runs_and_acts_step_by_step_as_in_a_window():
    torch, X = example()
    program = X.Program(envs=48, steps=20)
    losses = program.train(4)
    assert all(x == x and x >= 0 for x in losses)
    agreement, out, whole, states, last = program.act()
    assert 0 <= agreement <= 1
    assert float((out - whole).norm() / whole.norm()) <= 4e-4
    assert float((states - last).norm() / last.norm()) <= 4e-4


def reference(torch, st, x, tokens, starts, bins):
    """The student's logits by torch in double precision on the host."""
    p = {k: v.detach().double().cpu().requires_grad_() for k, v in st.named_parameters()}
    x, tokens, starts = x.double().cpu(), tokens.long().cpu(), starts.cpu()
    h, d = st.heads, st.dim
    linear = lambda name, y: y @ p[name + ".weight"].T + p[name + ".bias"]  # noqa: E731
    rms = lambda y, w=1.0: y / torch.sqrt((y * y).mean(-1, keepdim=True) + 1e-5) * w  # noqa: E731
    there = (tokens >= 0)[..., None]
    stream = linear("see", x) + st.act_dim ** -0.5 * (p["table"][tokens.clamp(min=0)] * there).sum(2)
    y = linear("inward", rms(stream, p["before"]))
    y, gate = y[..., :h * (3 * d + 2)].unflatten(-1, (h, 3 * d + 2)), y[..., h * (3 * d + 2):]
    q, k, v = (y[..., i * d:(i + 1) * d] for i in range(3))
    q, k = (torch.nn.functional.normalize(z, dim=-1) for z in (q, k))
    alpha = torch.where(starts[..., None], 0.0, torch.exp(-0.1 * torch.nn.functional.softplus(y[..., 3 * d])))
    beta = torch.sigmoid(y[..., 3 * d + 1])
    state, outs = torch.zeros(x.shape[0], h, d, d, dtype=torch.float64), []
    for t in range(x.shape[1]):
        state = alpha[:, t, :, None, None] * state
        u = beta[:, t, :, None] * (v[:, t] - (state * k[:, t, :, :, None]).sum(2))
        state = state + k[:, t, :, :, None] * u[:, :, None]
        outs.append(d ** -0.5 * (state * q[:, t, :, :, None]).sum(2))
    memory = rms(torch.stack(outs, 1)).flatten(-2) * p["heads_norm"] * gate * torch.sigmoid(gate)
    stream = stream + rms(linear("outward", memory), p["after"])
    u = rms(stream, p["ready"])
    a = u @ p["up_gate"].T
    stream = stream + rms((a * torch.sigmoid(a) * (u @ p["up"].T)) @ p["down"].T, p["last"])
    return linear("answer", rms(stream, p["final"])).view(-1, bins), p


def test_every_parameters_gradient_through_the_whole_student():
    torch, X = example()
    program = X.Program(envs=6, steps=9, seed=3)
    with torch.no_grad():                               # weights that are not all ones
        for w in program.student.parameters():
            w.add_(0.1 * torch.randn_like(w))
    state, starts = program.window()
    program.ask_teacher(state)
    x, tokens = program.seen(state), program.last_answers(starts)
    logits = program.student(x, tokens, starts)
    grad = torch.randn_like(logits)
    logits.backward(grad)
    want, p = reference(torch, program.student, x, tokens, starts, X.M.BINS)
    want.backward(grad.double().cpu())
    assert float((logits.detach().double().cpu() - want.detach()).norm() / want.detach().norm()) <= 4e-4
    for k, w in program.student.named_parameters():
        assert w.grad is not None, k
        assert float((w.grad.double().cpu() - p[k].grad).norm() / p[k].grad.norm()) <= 8e-4, k


def test_the_examples_functions_notice_changed_tensors_and_second_derivatives():
    torch, X = example()
    ctx = X.K.BlockContext()
    n = lambda *s: torch.randn(*s, device="cuda").requires_grad_()  # noqa: E731
    calls = [(lambda x, a, b, c: X.FeedForward.apply(ctx, "silu", x, a, b, c), lambda: [n(2, 3, 8), n(16, 8), n(16, 8), n(8, 16)]),
             (lambda x, y, g, w, p: sum(X.Residual.apply(ctx, 2, "silu", x, y, g, w, p)), lambda: [n(2, 3, 8), n(2, 3, 8), n(2, 3, 2), n(8), n(8)])]
    for f, inputs in calls:
        x = inputs()
        f(*x).sum().backward()
        assert all(t.grad is not None and bool(torch.isfinite(t.grad).all()) for t in x)
        for changed in range(len(x)):
            x = inputs()
            loss = f(*x).sum()
            with torch.no_grad():
                x[changed].mul_(2)
            with pytest.raises(RuntimeError, match="modified by an inplace operation"):
                loss.backward()
        x = inputs()
        first, = torch.autograd.grad(f(*x).square().sum(), x[0], create_graph=True)
        with pytest.raises(RuntimeError, match="once_differentiable"):
            first.sum().backward()


def test_acting_takes_the_kernels_for_few_rows_and_training_those_of_tiles():
    torch, X = example()
    program = X.Program(envs=48, steps=6)
    kernels = []
    for run in (program.act, lambda: program.train(1)):
        torch.cuda.synchronize()
        program.ctx.pql_profile_begin(4096)
        run()
        torch.cuda.synchronize()
        kernels.append({k["name"]: k["launches"] for k in program.ctx.pql_profile_end()})
    acted, trained = kernels
    assert acted["ffn_rows_kernel"] == 2 * program.steps        # every step; the window it is compared with has more rows
    assert "ffn_rows_kernel" not in trained and trained["ffn_gated_kernel"] == 1 and "ffn_back_kernel" in trained
