"""Orthogonalisation at the ends of its range: polynomials that are steep where the largest singular values are, norms far
below eps.

Tolerances of `check`: see test_orthogonalize_gpu.py.
"""
import numpy as np
import pytest
import torch

from matrices import DT, half, rounded
from oracle import step_oracle as oracle
from test_orthogonalize_gpu import check, make
from test_orthogonalize_range_cpu import STEEP

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(90, 140), (200, 150), (400, 700), (700, 400)])
def test_steep_polynomials(rows, cols, dtype):
    import paper_2410_10989_amd as flce
    print(f"case steep {rows} {cols} {dtype}", flush=True)
    G = make(rows, cols, dtype)
    got = flce.flce_orthogonalize([torch.from_numpy(G).to(DT[dtype]).cuda()], coefficients=STEEP)[0]
    torch.cuda.synchronize()
    check(got, G, dtype, coefficients=np.float32(STEEP).astype(float).tolist())


@pytest.mark.parametrize("ratio,eps,steps,scale", [(1e-4, 1e-7, 5, 1.0), (1e-8, 1e-7, 5, 1.0), (1e-12, 1e-7, 5, 1.0), (1e-4, 1.0, 12, 1.0),
                                                   (1e-30, 1.0, 5, 1.0), (1e-30, 1.0, 5, -3e20), (1e-9, 2.0 ** 100, 3, 1e10)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols,count", [(40, 60, 1), (150, 200, 1), (300, 400, 1), (400, 300, 1), (300, 700, 50)])
def test_norms_far_below_eps(rows, cols, count, dtype, ratio, eps, steps, scale):
    """|G| = ratio * eps: X is small from the first step on, and grows by a in each.  (At the mercy of one power of two for all
    matrices it vanished.)  Tolerance, relative to the norm: B = a I, X and the products' sums are rounded in each step.
    Operands in one plane (bf16 of more than 256 rows; in the Gram product any bf16, which counts where X gets large,
    in the last of 12 steps): 2^-11 each for B and X; in two: 2^-21 each, 2^-21 for the product of the lo planes and the sums.
    The result is rounded once."""
    import paper_2410_10989_amd as flce
    print(f"case {rows} {cols} {dtype} ratio {ratio} eps {eps}", flush=True)
    G = make(rows, cols, dtype)
    G = rounded(G * (ratio * eps / np.linalg.norm(G)), dtype)
    eps, scale = float(np.float32(eps)), float(np.float32(scale))
    ts = [torch.from_numpy(G).to(DT[dtype]).cuda() for _ in range(count)]
    got = flce.flce_orthogonalize(ts, eps=eps, steps=steps, scale=scale)[-1].double().cpu().numpy()
    ref = oracle.orthogonalize(G, eps=eps, steps=steps, scale=scale, coefficients=np.float32(oracle.COEFFICIENTS).astype(float))
    one_plane = dtype == "bf16" and (min(rows, cols) > 256 or steps == 12)
    off, may = np.linalg.norm(got - ref) / np.linalg.norm(ref), steps * (2.0 ** -10 if one_plane else 3 * 2.0 ** -21) + half(dtype)
    print(f"off {off:.2e}, may be {may:.2e}", flush=True)
    assert np.linalg.norm(ref) > 0 and off <= may


def test_a_list_of_norms_on_either_side_of_eps():
    """Each matrix has powers of two of its own, and the result is that of the matrix alone."""
    import paper_2410_10989_amd as flce
    for rows, cols in ((60, 40), (300, 400)):
        ts = [torch.from_numpy(make(rows, cols, "f32", seed=i)).float().cuda() * 10.0 ** -i for i in range(0, 24, 3)]
        want = [flce.flce_orthogonalize([t], outs=[torch.empty_like(t)], eps=1e-6)[0] for t in ts]
        zero = torch.zeros_like(ts[0])
        got = flce.flce_orthogonalize(ts + [zero], outs=[torch.empty_like(t) for t in ts + [zero]], eps=1e-6)
        for g, w, t in zip(got, want, ts):
            ref = oracle.orthogonalize(t.double().cpu().numpy(), eps=float(np.float32(1e-6)))
            for o in (g, w):   # (they may be cut into other ranges of K)
                assert np.linalg.norm(o.double().cpu().numpy() - ref) <= 5 * 3 * 2.0 ** -21 * np.linalg.norm(ref)
        assert (got[-1] == 0).all()
