"""The example that runs the student's operators together.

Tolerance: outputs and states by steps and as one window are each within 1e-5 (2-norm) of the exact result, the bound
their own tests derive, so they are within 2e-5 of each other."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu


def test_a_student_learns_and_acts():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible: the gpu-marked tests need a real MI355X")
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import memory_student
    program = memory_student.Program(envs=64, steps=40)
    before = program.act()[0]
    losses = program.train(60)
    assert all(x == x and x >= 0 for x in losses)
    assert sum(losses[-10:]) < sum(losses[:10])
    after, out, whole, states, last = program.act()
    assert after > before
    assert float((out - whole).norm() / whole.norm()) <= 2e-5
    assert float((states - last).norm() / last.norm()) <= 2e-5


def test_the_examples_function_notices_changed_tensors_and_second_derivatives():
    import torch
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import memory_student as M
    ctx = M.S.StudentContext()

    def inputs():
        g = torch.Generator(device="cuda").manual_seed(3)
        q, k, v = (torch.randn(2, 6, 1, 8, device="cuda", generator=g).requires_grad_() for _ in range(3))
        decay = -torch.rand(2, 6, 1, device="cuda", generator=g)
        return q, k, v, decay.requires_grad_(), torch.rand(2, 6, 1, device="cuda", generator=g).requires_grad_()
    x = inputs()
    M.DeltaRule.apply(ctx, *x).sum().backward()
    assert all(t.grad is not None and torch.isfinite(t.grad).all() for t in x)
    for changed in range(5):
        x = inputs()
        loss = M.DeltaRule.apply(ctx, *x).sum()
        with torch.no_grad():
            x[changed].mul_(2)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.backward()
    x = inputs()
    first, = torch.autograd.grad(M.DeltaRule.apply(ctx, *x).square().sum(), x[2], create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        first.sum().backward()
