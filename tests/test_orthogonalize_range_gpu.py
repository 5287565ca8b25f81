"""Orthogonalisation at the ends of its range: polynomials that are steep where the largest singular values are.

Tolerances of `check`: see test_orthogonalize_gpu.py.
"""
import numpy as np
import pytest
import torch

from matrices import DT
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
