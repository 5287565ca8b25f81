"""Layer norm of rows that lie far from zero, and of rows of equal elements.

Tolerances, element by element, with p the rounded mean, q the mean of h - p, d = h - mean, r = 1 / sqrt(var + eps), xh = d r.
A sum over a row is off by at most (16 + H / 1024 + 16) 2^-24 <= 2^-18 of its magnitudes for H <= 32768 (see
test_layer_norm_gpu.py), so |q| <= 2^-18 mean |h|, and q is off by 2^-18 mean |h - p| <= 2^-18 mean |d| + 2^-36 mean |h|; h - p
has one rounding of itself, and the variance is off by 2^-18 (1 + q^2 / var) of itself, whose second term is below 1 here.  That
is 2^-17 (|xh| + mean |xh|) + 2^-36 mean |h| r for xh; where h = x + y, its rounding, 2^-24 |h| r, comes on top.  The other
factors are those of test_layer_norm_gpu.py.  In them nothing of the size of 2^-24 |h| r is left, which is up to 300 times
what is asked for here of rows of 100.
"""
import numpy as np
import pytest
import torch

from matrices import DT, half, rounded
from oracle import step_oracle as oracle

pytestmark = pytest.mark.gpu

ARITH = 2.0 ** -17
TINY = 2.0 ** -126


def magnitudes(h, eps):
    """xh, and what its error is 2^-17 of."""
    d = h - h.mean(1, keepdims=True)
    r = 1 / np.sqrt((d * d).mean(1, keepdims=True) + eps)
    return d * r, r, (np.abs(d) + np.abs(d).mean(1, keepdims=True) + 2.0 ** -19 * np.abs(h).mean(1, keepdims=True)) * r


def inside(name, got, ref, slack, mag, dtype):
    got = got.double().cpu().numpy()
    over = np.abs(got - ref) - (half(dtype) * (1 + slack) * np.abs(ref) + slack * (1 + half(dtype)) * mag + TINY)
    at = np.unravel_index(over.argmax(), over.shape)
    assert np.isfinite(got).all() and over.max() <= 0, f"{name}{at}: {got[at]!r} instead of {ref[at]!r}"


def rows_of(kind, rows, H, dtype, g):
    level = 100.0 * np.exp(g.standard_normal((rows, 1)))
    if kind == "equal":
        return rounded(np.repeat(level, H, 1), dtype)
    return rounded(level + level * kind * g.standard_normal((rows, H)), dtype)   # kind: the deviation, of the level


CASES = [("equal", 300, 33), ("equal", 300, 100), ("equal", 200, 513), ("equal", 300, 1000), ("equal", 100, 2050), ("equal", 300, 4096),
         ("equal", 60, 5000), ("equal", 60, 12001), ("equal", 20, 20001), ("equal", 50, 5), (1e-3, 100, 1000), (1e-3, 50, 4096),
         (1e-4, 100, 515), (1e-4, 40, 8192), (1e-4, 10, 20000), (1e-2, 77, 136)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind,rows,H", CASES)
def test_far_from_zero(kind, rows, H, dtype):
    import paper_2410_10989_amd as flce
    print(f"case {kind} {rows} {H} {dtype}", flush=True)
    g = np.random.Generator(np.random.Philox(key=[rows, H]))
    h, eps = rows_of(kind, rows, H, dtype, g), float(np.float32(1e-5))
    gamma, beta = rounded(1 + 0.2 * g.standard_normal(H), dtype), rounded(0.3 * g.standard_normal(H), dtype)
    dn, dh = rounded(0.02 * g.standard_normal((rows, H)), dtype), rounded(0.01 * g.standard_normal((rows, H)), dtype)
    put = lambda a: torch.from_numpy(a).to(DT[dtype]).cuda()
    xh, r, mag = magnitudes(h, eps)
    n = flce.flce_layer_norm_fwd(put(h), gamma=put(gamma), beta=put(beta), eps=eps)[1]
    ref = oracle.layer_norm(h, None, gamma, beta, eps)
    inside("n", n, ref["n"], ARITH, np.abs(gamma) * mag + np.abs(gamma * xh) + np.abs(beta), dtype)
    got = flce.flce_layer_norm_bwd(put(h), put(dn), put(dh), put(gamma), True, eps)
    ref = oracle.layer_norm_grad(h, dn, dh, gamma, eps)
    u, xm = dn * gamma, np.abs(xh) + mag
    dx_mag = np.abs(dh) + r * (np.abs(u) + np.abs(u).mean(1, keepdims=True) + 2 * xm * (np.abs(u) * xm).mean(1, keepdims=True))
    inside("dx", got[0], ref["dx"], ARITH, dx_mag, dtype)
    rows_slack = ARITH + (rows + 32) * 2.0 ** -24
    inside("dgamma", got[1][None], ref["dgamma"][None], rows_slack, (np.abs(dn) * xm).sum(0)[None], dtype)
    inside("dbeta", got[2][None], ref["dbeta"][None], rows_slack, np.abs(dn).sum(0)[None], dtype)


@pytest.mark.parametrize("rows,H", [(40, 1000), (9, 4100), (5, 20000)])
def test_a_residual_that_takes_the_offset_away(rows, H):
    """x far from zero, y nearly -x: h = x + y is exact in fp32 (both are multiples of 2^-16 below 2^8), and so is n to its
    own accuracy."""
    import paper_2410_10989_amd as flce
    g = np.random.Generator(np.random.Philox(key=[rows, H + 1]))
    x = np.round(200 * 2 ** 16 + 2 ** 16 * g.standard_normal((rows, H))) / 2 ** 16
    y = np.round(-200 * 2 ** 16 + 2 ** 10 * g.standard_normal((rows, H))) / 2 ** 16
    h, n = flce.flce_layer_norm_fwd(torch.from_numpy(x).float().cuda(), torch.from_numpy(y).float().cuda(), eps=1e-5)
    assert torch.equal(h.double().cpu(), torch.from_numpy(x + y))
    xh, r, mag = magnitudes(x + y, float(np.float32(1e-5)))
    inside("n", n, oracle.layer_norm(x, y, eps=float(np.float32(1e-5)))["n"], ARITH, mag + np.abs(xh), "f32")
