"""Orthogonalisation of matrices up to the largest that are taken, against the same steps in 64 bits on the GPU.

Tolerances.  fp32 matrices: what fp32 arithmetic (torch's own products) is off by on the same matrix, which the operands' 22 bits
and fp32 sums are to stay below, and 2^-21.  bf16: operands of 11 bits, of which B and X are rounded in each step, 2^-11 each, and
one rounding of the result.
"""
import pytest
import torch

from matrices import DT, half

pytestmark = pytest.mark.gpu

A, B, C = torch.tensor([3.4445, -4.7750, 2.0315]).double().tolist()


def steps(X):
    X = X / (torch.linalg.vector_norm(X) + 1e-7)
    for _ in range(5):
        G = torch.mm(X, X.t().contiguous())
        X = A * X + torch.mm(B * G + C * torch.mm(G, G), X)
    return X


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols,count", [(4096, 4096, 1), (4096, 14336, 1), (14336, 4096, 1), (16384, 16384, 1), (100, 1 << 20, 1),
                                             (1 << 20, 100, 1), (1, 1 << 20, 1), (64, 1 << 18, 130), (2048, 2048, 4), (1024, 2048, 14)])
def test_large(rows, cols, count, dtype):
    import paper_2410_10989_amd as flce
    print(f"case {count} {rows} {cols} {dtype}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(rows + cols)
    t = (1e-3 * torch.randn(rows, cols, device="cuda", generator=g)).to(DT[dtype])
    outs = [torch.empty_like(t) for _ in range(count)]
    flce.flce_orthogonalize([t] * count, outs=outs)
    wide = t if rows <= cols else t.t().contiguous()
    ref = steps(wide.double())
    size = torch.linalg.vector_norm(ref).item()
    off = lambda x: torch.linalg.vector_norm((x if rows <= cols else x.t()).double() - ref).item() / size
    plain = torch.linalg.vector_norm(steps(wide.float()).double() - ref).item() / size if dtype == "f32" else 0.0
    may = plain + 2.0 ** -21 if dtype == "f32" else 5 * 2.0 ** -10 + half(dtype)
    for o in (outs[0], outs[-1]):
        print(f"off {off(o):.2e}, may be {may:.2e}", flush=True)
        assert o.isfinite().all() and off(o) <= may
    # (the first ones and the last may be cut into other ranges of K)
    assert all(torch.equal(o, outs[0]) for o in outs[:count // 2])
