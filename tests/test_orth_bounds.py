"""The tolerances that the update's GPU tests use, on the CPU: mistakes planted in the reference fall outside them, the same
steps with operands in two 11-bit parts inside.
"""
import numpy as np
import pytest

import oracle.model_oracle as M

from .test_gpu_orth_values import COEF, EPS, exact

F32 = [float(np.float32(c)) for c in COEF]


def matrix(kind, rows, cols, seed):
    rng = np.random.default_rng(seed)
    if kind == "rank 1":
        x = rng.normal(size=(rows, 1)) @ rng.normal(size=(1, cols))
    elif kind == "twice":
        x = np.tile(rng.normal(size=((rows + 1) // 2, cols)), (2, 1))[:rows]
    else:
        x = rng.normal(size=(rows, cols)) * (np.logspace(0, -3, cols) if kind == "steep" else 1e-3)
    return x.astype(np.float32).astype(np.float64)


def in_parts(x, bits, n):
    """x as the sum of n parts of so many bits."""
    got = np.zeros_like(x)
    for _ in range(n):
        m, e = np.frexp(x - got)
        got = got + np.ldexp(np.round(np.ldexp(m, bits)), e - bits)
    return got


def steps_in_parts(g, steps, bits, n):
    a, b, c = F32
    x = g / (np.linalg.norm(g) + EPS)
    tall = x.shape[0] > x.shape[1]
    x = in_parts(x.T if tall else x, bits, n)
    for _ in range(steps):
        gram = in_parts(x @ x.T, bits, n)
        x = in_parts(a * x + in_parts(b * gram + c * (gram @ gram), bits, n) @ x, bits, n)
    return x.T if tall else x


@pytest.mark.parametrize("rows,cols", [(96, 160), (80, 1000), (400, 72), (40, 90)])
@pytest.mark.parametrize("kind", ["broad", "steep", "rank 1", "twice"])
def test_planted_mistakes_fall_outside(rows, cols, kind):
    g = matrix(kind, rows, cols, 1)
    want, tol = exact(g, 5, COEF)
    assert tol < 0.05 * np.linalg.norm(want)
    inside = steps_in_parts(g, 5, 11, 2)
    if min(rows, cols) > 64:
        assert np.linalg.norm(inside - want) <= tol
    mistakes = {
        "zeros": np.zeros_like(want),
        "another matrix's": exact(matrix(kind, rows, cols, 2), 5, COEF)[0],
        "a step fewer": exact(g, 4, COEF)[0],
        "b off by a thousandth": M.newton_schulz(g, 5, F32[0], F32[1] * 1.001, F32[2], EPS)[0],
        "turned around": -want,
        "operands of 11 bits": steps_in_parts(g, 5, 11, 1),
        "a row left out": np.concatenate([np.zeros_like(want[:1]), want[1:]]),
    }
    for name, wrong in mistakes.items():
        assert np.linalg.norm(wrong - want) > tol, name
