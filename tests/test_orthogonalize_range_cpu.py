"""Which polynomials the orthogonalisation takes: those that keep every singular value of [0, 1] at 1024 or below, as
exact arithmetic says, however steep they are where the largest of them are."""
import ctypes

import numpy as np
import pytest

import paper_2410_10989_amd as flce

# Five steps for singular values of [0, 1], steep at their upper end: the largest value after each is 1.992, 1.966, 1.866,
# 1.560, 1.124, but 1.01 in the place of 1 becomes 8866 in four of them.
STEEP = [(8.2872, -23.5959, 17.3004), (4.1071, -2.9478, 0.5448), (3.9487, -2.9089, 0.5518), (3.3184, -2.4885, 0.5100), (2.3007, -1.6689, 0.4188)]


def largest(coefficients):
    """The largest singular value after each step: over a fine grid of [0, 1], in 64 bits."""
    x = np.linspace(0.0, 1.0, 2_000_001)
    most = []
    for a, b, c in np.float32(coefficients).astype(np.float64):
        x = np.abs(a * x + b * x ** 3 + c * x ** 5)
        most.append(x.max())
    return most


def taken(coefficients, steps, dtype, rows=70, cols=90):
    flat = (ctypes.c_float * (3 * steps))(*[v for c in coefficients[:steps] for v in c])
    a = flce.FlceOrthogonalizeArgs(ctypes.sizeof(flce.FlceOrthogonalizeArgs), rows, cols, dtype, steps, ctypes.addressof(flat), 1, 1.0, 1e-7)
    return flce.lib().flce_orthogonalize_workspace_bytes(1, ctypes.byref(a)) > 0


@pytest.mark.parametrize("dtype", [flce.FLCE_F32, flce.FLCE_BF16])
@pytest.mark.parametrize("rows,cols", [(70, 90), (200, 300), (400, 700)])
@pytest.mark.parametrize("steps", [1, 2, 3, 4, 5])
def test_steep_polynomials_are_taken(steps, rows, cols, dtype):
    assert max(largest(STEEP[:steps])) < 2.0
    assert taken(STEEP, steps, dtype, rows, cols)


@pytest.mark.parametrize("dtype", [flce.FLCE_F32, flce.FLCE_BF16])
def test_the_limit_is_where_it_is_said_to_be(dtype):
    for first, last in [((31.9, 0.0, 0.0), (32.0, 0.0, 0.0)), ((1.0, 0.0, 0.0), (1024.0, 0.0, 0.0)), ((0.0, 0.0, 2.0), (0.0, 0.0, 31.99))]:
        assert max(largest([first, last])) <= 1024.0 and taken([first, last], 2, dtype)
    for first, last in [((32.1, 0.0, 0.0), (32.0, 0.0, 0.0)), ((1.0, 0.0, 0.0), (1024.5, 0.0, 0.0)), ((0.0, 0.0, 2.0), (0.0, 0.0, 32.01))]:
        assert max(largest([first, last])) > 1024.0 and not taken([first, last], 2, dtype)


def test_polynomials_at_random():
    """Either side of the limit, by the grid's largest value; nothing is said where that is within 1e-5 of it."""
    g = np.random.Generator(np.random.Philox(key=[7, 8]))
    sides = [0, 0]
    for _ in range(150):
        steps = int(g.integers(1, 5))
        c = (g.standard_normal((steps, 3)) * np.exp(g.uniform(0.0, 2.5, (steps, 1)))).astype(np.float32).astype(float)
        most = max(largest(c))
        if abs(most - 1024.0) < 1e-2:
            continue
        assert taken(c.tolist(), steps, flce.FLCE_F32) == (most < 1024.0), (c, most)
        sides[int(most < 1024.0)] += 1
    assert min(sides) > 10
