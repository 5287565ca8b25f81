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


USUAL = [oracle.COEFFICIENTS] * 5
FALLING = [(4.0848, -6.8946, 2.9270), (3.9505, -6.3029, 2.6377), (3.7418, -5.5913, 2.3037), (2.8769, -3.1427, 1.2046), (2.8366, -3.0525, 1.2012)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("spike", [0.0, 30.0, 100.0, 300.0])
@pytest.mark.parametrize("rows,cols", [(300, 700), (700, 300)])
@pytest.mark.parametrize("coefficients", [USUAL, FALLING, [(8.0, -22.0, 16.0)] * 2], ids=["usual", "falling", "steep"])
def test_long_lists_of_long_matrices(coefficients, rows, cols, spike, dtype):
    """A list that fills the chip takes two steps at a time where its matrices are long.  Low rank and noise: that may cost half
    as much again as the matrix alone is off by, and no more, whatever the coefficients are.

    Tolerances are of the 2-norm, that of `check` among them.  Its bar for single elements is four times the largest of another
    sample, which holds for errors that are alike in all elements; here they lie along the large singular vectors, u_i v_j
    times what two directions are off by, so the largest may be any share of the 2-norm, and its square is at most the sum of
    all squares, which is bounded here."""
    import paper_2410_10989_amd as flce
    G = make(rows, cols, dtype, rank=2 if spike else 0, spike=spike)
    c = np.float32(coefficients).astype(float).tolist()
    t = torch.from_numpy(G).to(DT[dtype]).cuda()
    ref = oracle.orthogonalize(G, steps=len(c), coefficients=c)
    model = oracle.orthogonalize_rounded(G, 2 if dtype == "f32" else 1, steps=len(c), coefficients=c)
    size = np.linalg.norm(ref)
    off = []
    for count in (1, 50):
        got = flce.flce_orthogonalize([t] * count, outs=[torch.empty_like(t) for _ in range(count)], steps=len(c), coefficients=c)[-1]
        off.append(np.linalg.norm(got.double().cpu().numpy() - ref) / size)
    may = 2 * np.linalg.norm(model - ref) / size + half(dtype) + 2.0 ** -21
    print(f"alone {off[0]:.2e}, in a list {off[1]:.2e}, may be {may:.2e}", flush=True)
    assert max(off) <= may
    # (fp32: two samples of roundings at the end of fp32, 2^-21 apart at the most)
    assert off[1] <= 1.5 * off[0] + 2.0 ** -21


@pytest.mark.parametrize("second", [0.0, 0.01])
@pytest.mark.parametrize("rows,cols", [(60, 100), (100, 60), (120, 128), (20, 500), (200, 300)])
@pytest.mark.parametrize("coefficients", [USUAL, FALLING, [(8.0, -22.0, 16.0)] * 2, [(1.5, -0.5, 0.0)] * 8], ids=["usual", "falling", "steep", "cubic"])
def test_small_matrices_of_rank_one_and_two(coefficients, rows, cols, second, dtype="bf16"):
    """What is left of such a matrix in all other directions is its rounding to bf16, which all steps lift: those that
    a small matrix takes in one launch are to be as good as one by one.  Of the 2-norm, for the reason in
    test_long_lists_of_long_matrices.

    The steep steps take a singular value of 1 to 2 and 352, which is beyond the model's one scale of 2^13.  Where it
    overflows: with l = x^2 off by 2^-11 of itself (A in one plane), x (a + b l + c l^2) is off by |b l + 2 c l^2| / |a + b l +
    c l^2| of that, 10 / 2 of it at l = 1 and 424 / 176 at l = 4, where an error of x counts |a + 3 b l + 5 c l^2| / 176 = 5.82
    times: 5 * 5.82 + 2.41 < 32 times 2^-11 in all."""
    import paper_2410_10989_amd as flce
    print(f"case {rows} {cols} {second}", flush=True)
    g = np.random.Generator(np.random.Philox(key=[rows, cols]))
    outer = lambda: np.outer(g.standard_normal(rows), g.standard_normal(cols))
    G = rounded(outer() + second * outer(), dtype)
    c = np.float32(coefficients).astype(float).tolist()
    got = flce.flce_orthogonalize([torch.from_numpy(G).to(DT[dtype]).cuda()], steps=len(c), coefficients=c)[0].double().cpu().numpy()
    ref = oracle.orthogonalize(G, steps=len(c), coefficients=c)
    with np.errstate(over="ignore", invalid="ignore"):
        model = oracle.orthogonalize_rounded(G, 1, steps=len(c), coefficients=c)
    lost = np.linalg.norm(model - ref) / np.linalg.norm(ref)
    off, may = np.linalg.norm(got - ref) / np.linalg.norm(ref), (2 * lost if np.isfinite(lost) else 32 * 2.0 ** -11) + half(dtype) + 2.0 ** -21
    print(f"off {off:.2e}, may be {may:.2e}", flush=True)
    assert off <= may
