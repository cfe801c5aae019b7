"""A student made of a block around its memory: python examples/block_student.py

The task and the teacher are those of memory_student.py.  This student also reads its last answers, as tokens, and its
memory stands in a block: norms before and after it with a gate and a residual sum, and a gated feed-forward block.

  tokens     pql_embed_forward: the last answers' bins, one for each action dimension, added to a projection of what is seen
  memory     pql_residual_forward (norm), torch's projections, pql_delta_forward, pql_residual_forward (a norm for each head
             and its gate), the sum with the residual stream and the next norm in another
  block      pql_ffn_forward, and the last sum and norm

Training goes through every call's gradient; acting runs the same calls for one step of all environments at a time.  Episodes end
where the memory is told to forget.
"""
from __future__ import annotations

import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

import torch  # noqa: E402

import memory_student as M  # noqa: E402
from paper_2307_12983_amd import block as K  # noqa: E402
from paper_2307_12983_amd import student as S  # noqa: E402

EPS = 1e-5


def rows(t):
    return None if t is None else K.Rows(t)


class Embed(torch.autograd.Function):
    """scale times the sum of a row's tokens' embeddings."""

    @staticmethod
    def forward(fn, ctx, tokens, table, scale):
        shape = K.embed_shape(tokens, table, scale)
        out = table.new_empty(*tokens.shape[:2], table.shape[1])
        ctx.pql_embed_forward(shape, tokens, None, K.Rows(table), K.Rows(out))
        fn.call = ctx, shape
        fn.save_for_backward(tokens, table)
        return out

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(fn, out_grad):
        ctx, shape = fn.call
        tokens, table = fn.saved_tensors
        grad = torch.empty_like(table)
        ctx.pql_embed_backward(shape, tokens, None, K.Rows(out_grad.contiguous()), K.Rows(grad), K.workspace(ctx.embed_workspace_bytes(shape)))
        return None, None, grad, None


class Residual(torch.autograd.Function):
    """pql_residual_forward: the sum (None if it has no norm after it), and its norm (None without x or pre)."""

    @staticmethod
    def forward(fn, ctx, groups, act, x, y, gate, post, pre):
        like = x if x is not None else y
        shape = K.residual_shape(*like.shape, like.dtype, groups, 0 if gate is None else gate.shape[-1], act,
                                 EPS if post is not None else 0.0, EPS if pre is not None else 0.0)
        given = K.ResidualInput(shape, x, y, gate, post, pre)
        total = None if y is None else torch.empty_like(like)
        after = None if pre is None else torch.empty_like(like)
        ctx.pql_residual_forward(shape, given, rows(total), rows(after))
        fn.call = ctx, shape
        fn.save_for_backward(x, y, gate, post, pre)
        return total, after

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(fn, total_grad, after_grad):
        ctx, shape = fn.call
        given = fn.saved_tensors
        grads = [None if t is None else torch.empty_like(t) for t in given]
        dense = [None if g is None else g.contiguous() for g in (total_grad, after_grad)]
        ctx.pql_residual_backward(shape, K.ResidualInput(shape, *given), rows(dense[0]), rows(dense[1]), K.ResidualGrad(shape, *grads),
                                  K.workspace(ctx.residual_workspace_bytes(shape)))
        return (None, None, None, *grads)


def feed_forward(ctx, act, x, gate, up, down, keep):
    """The block's result, and what its gradient is worked out from: without it, calls of few rows take kernels of their own."""
    shape = K.ffn_shape(x, gate, act)
    out = torch.empty_like(x)
    saved = K.workspace(ctx.ffn_saved_bytes(shape)) if keep else None
    ctx.pql_ffn_forward(shape, K.FfnInput(shape, x, gate, up, down), K.Rows(out), saved, K.workspace(ctx.ffn_workspace_bytes(shape, K.FFN_FORWARD)))
    return out, saved, shape


class FeedForward(torch.autograd.Function):
    @staticmethod
    def forward(fn, ctx, act, x, gate, up, down):
        out, saved, shape = feed_forward(ctx, act, x, gate, up, down, any(t.requires_grad for t in (x, gate, up, down)))
        fn.call = ctx, shape
        fn.save_for_backward(x, gate, up, down, saved)
        return out

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(fn, out_grad):
        ctx, shape = fn.call
        *given, saved = fn.saved_tensors
        grads = [torch.empty_like(t) for t in given]
        call = K.FFN_BACKWARD if saved is not None else K.FFN_BACKWARD_ALONE
        ctx.pql_ffn_backward(shape, K.FfnInput(shape, *given), saved, K.Rows(out_grad.contiguous()), K.FfnGrad(shape, *grads),
                             K.workspace(ctx.ffn_workspace_bytes(shape, call)))
        return (None, None, *grads)


class BlockStudent(torch.nn.Module):
    def __init__(self, ctx, seen, act_dim, heads=4, dim=32, hidden=256):
        super().__init__()
        self.ctx, self.heads, self.dim, self.act_dim, self.width = ctx, heads, dim, act_dim, heads * dim
        w = self.width
        weight = lambda *s: torch.nn.Parameter(torch.randn(*s) * s[-1] ** -0.5)  # noqa: E731
        ones = lambda n: torch.nn.Parameter(torch.ones(n))  # noqa: E731
        self.table = torch.nn.Parameter(torch.randn(act_dim * M.BINS, w) * 0.1)
        self.see = torch.nn.Linear(seen, w)
        self.before, self.heads_norm, self.after, self.ready, self.last, self.final = (ones(w) for _ in range(6))
        self.inward = torch.nn.Linear(w, heads * (3 * dim + 2) + w)         # q, k, v, decay, beta and the heads' gate
        self.outward = torch.nn.Linear(w, w)
        self.up_gate, self.up, self.down = weight(hidden, w), weight(hidden, w), weight(w, hidden)
        self.answer = torch.nn.Linear(w, act_dim * M.BINS)

    def enter(self, x, tokens):
        """The residual stream: what is seen and the last answers."""
        return self.see(x) + Embed.apply(self.ctx, tokens, self.table, self.act_dim ** -0.5)

    def tokens(self, stream, starts):
        """q, k, v, log_decay, beta of the memory and its gate."""
        h, d = self.heads, self.dim
        y = self.inward(Residual.apply(self.ctx, 1, "none", stream, None, None, None, self.before)[1])
        y, gate = y[..., :h * (3 * d + 2)].unflatten(-1, (h, 3 * d + 2)), y[..., h * (3 * d + 2):].contiguous()
        q, k, v = (y[..., i * d:(i + 1) * d] for i in range(3))
        decay = (-0.1 * torch.nn.functional.softplus(y[..., 3 * d])).masked_fill(starts[..., None], -float("inf"))
        norm = torch.nn.functional.normalize
        return [t.contiguous() for t in (norm(q, dim=-1), norm(k, dim=-1), v, decay, torch.sigmoid(y[..., 3 * d + 1]))], gate

    def leave(self, stream, memory, gate):
        """Behind the memory: logits of every step and action dimension."""
        y, _ = Residual.apply(self.ctx, self.heads, "silu", None, memory.flatten(-2), gate, self.heads_norm, None)
        stream, u = Residual.apply(self.ctx, 1, "none", stream, self.outward(y), None, self.after, self.ready)
        block = self.ctx, "silu", u, self.up_gate, self.up, self.down
        f = FeedForward.apply(*block) if torch.is_grad_enabled() else feed_forward(*block, keep=False)[0]
        _, u = Residual.apply(self.ctx, 1, "none", stream, f, None, self.last, self.final)
        return self.answer(u).view(-1, M.BINS)

    def forward(self, x, tokens, starts):
        stream = self.enter(x, tokens)
        given, gate = self.tokens(stream, starts)
        return self.leave(stream, M.DeltaRule.apply(self.ctx, *given), gate)


class Program(M.Program):
    """The program of memory_student.py with this student; its last answers are the teacher's, one step late."""

    def __init__(self, envs=256, steps=24, seed=0):
        super().__init__(envs, steps, seed)
        self.ctx = K.BlockContext()
        torch.manual_seed(seed)
        self.student = BlockStudent(self.ctx, 2 * self.w.obs_dim, self.w.act_dim).cuda()
        self.adam = torch.optim.Adam(self.student.parameters(), lr=3e-3)

    def last_answers(self, starts):
        """Tokens [envs, steps, act_dim]: the bins answered one step before, none at an episode's start."""
        bins = self.teacher.index[:, 0].view(self.envs, self.steps, -1)
        tokens = bins + M.BINS * torch.arange(self.w.act_dim, dtype=torch.int32, device="cuda")
        tokens = torch.cat([torch.full_like(tokens[:, :1], -1), tokens[:, :-1]], 1)
        return tokens.masked_fill(starts[..., None], -1).contiguous()

    def train(self, iterations, report=None):
        losses = []
        for i in range(iterations):
            state, starts = self.window()
            self.ask_teacher(state)
            logits = self.student(self.seen(state), self.last_answers(starts), starts)
            grad = torch.empty_like(logits)
            self.ctx.pql_distill_loss(S.Logits(logits.detach()), self.teacher, 1.0, self.weight, self.loss, self.lse, S.Logits(grad),
                                      self.space)
            self.adam.zero_grad(set_to_none=True)
            logits.backward(grad)
            self.adam.step()
            losses.append(self.loss.sum())
            if report and (i + 1) % report == 0:
                print("iteration %4d  loss %.4f" % (i + 1, float(losses[-1])), flush=True)
        return [float(x) for x in losses]

    @torch.no_grad()
    def act(self):
        """The student step by step over a window.  Returns how often its first answer is the teacher's at the last step of each
        window, its logits by steps and as one window, and the memory's states after both."""
        state, starts = self.window()
        self.ask_teacher(state)
        x, tokens, st = self.seen(state), self.last_answers(starts), self.student
        states = torch.zeros(self.envs, st.heads, st.dim, st.dim, device="cuda")
        logits = []
        for t in range(self.steps):
            s = slice(t, t + 1)
            stream = st.enter(x[:, s], tokens[:, s].contiguous())
            given, gate = st.tokens(stream, starts[:, s])
            out = torch.empty_like(given[2])
            self.ctx.pql_delta_step(S.delta_shape(given[0], given[2], st.dim ** -0.5), S.DeltaInput(*given, state=states), states, S.Sequence(out))
            logits.append(st.leave(stream, out, gate).view(self.envs, 1, st.act_dim, M.BINS))
        logits = torch.cat(logits, 1)
        stream = st.enter(x, tokens)
        given, gate = st.tokens(stream, starts)
        out, last = torch.empty_like(given[2]), torch.empty_like(states)
        shape = S.delta_shape(given[0], given[2], st.dim ** -0.5)
        self.ctx.pql_delta_forward(shape, S.DeltaInput(*given), S.Sequence(out), last, None, S.workspace(self.ctx.delta_workspace_bytes(shape, False)))
        whole = st.leave(stream, out, gate).view_as(logits)
        answer = logits[:, -1].argmax(-1).flatten()
        teacher = self.teacher.index[:, 0].view(self.envs, self.steps, -1)[:, -1].flatten()
        return float((answer == teacher).float().mean()), logits, whole, states, last


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--envs", type=int, default=256)
    p.add_argument("--steps", type=int, default=24, help="steps of a window")
    p.add_argument("--iterations", type=int, default=300)
    a = p.parse_args(argv)
    program = Program(a.envs, a.steps)
    print("first answers that are the teacher's: %.3f untrained" % program.act()[0])
    program.train(a.iterations, max(1, a.iterations // 10))
    agreement, out, whole, states, last = program.act()
    off = lambda x, y: float((x - y).norm() / y.norm())  # noqa: E731
    print("first answers that are the teacher's: %.3f trained" % agreement)
    print("step by step against one window: logits off by %.1e, states by %.1e" % (off(out, whole), off(states, last)))


if __name__ == "__main__":
    main()
