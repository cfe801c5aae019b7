"""The student's operators where values, sizes or counts come to the limits of what the calls take, against the
double-precision reference.  Tolerances: those of test_gpu_student.py, derived there."""
import numpy as np
import pytest

from test_gpu_student import Delta, close, env  # noqa: F401

pytestmark = pytest.mark.gpu
GRADS = ("dq", "dk", "dv", "dg", "dbeta", "dstate")
LOWEST = float(np.finfo(np.float32).min)


def held(x):
    """What 32 bits hold of a value: nothing below half their smallest number."""
    return np.where(np.abs(x) < 2.0 ** -150, 0.0, x)


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
