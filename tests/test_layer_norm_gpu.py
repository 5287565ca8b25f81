"""Layer norm with the residual sum in front of it (forward and backward) against its 64-bit definition.

Tolerances, element by element: half a step of the storage type of the value (one rounding of the output), plus
2^-17 of the magnitude of what was added up to it (`_mag` of the definition).  The latter covers fp32 arithmetic: a row's
sums (at most 16 terms one after the other per thread, or H / 1024 in the long form, then a tree) are off by less than
(16 + H / 1024 + 16) 2^-24 <= 2^-18 of their magnitudes for H <= 32768; the mean's error enters h - mean (the magnitudes
hold |h| and its mean for that), the squares' half as much after the root, and the two row sums of the backward
with the factors they meet; up to a dozen factors of 2^-24 each.  Sums over rows: one more 2^-24 of the terms'
magnitudes per row and partial sum.
"""
import numpy as np
import pytest
import torch

from matrices import DT, Matrix, half, rounded
from oracle import step_oracle as oracle

pytestmark = pytest.mark.gpu

ARITH = 2.0 ** -17
TINY = 2.0 ** -126


def check(name, got, ref, dtype, rows=0):
    value, mag = ref[name], ref[name + "_mag"]
    got = got.double().cpu().numpy()
    assert got.shape == value.shape and np.isfinite(got).all(), name
    slack = ARITH + (rows + 32) * 2.0 ** -24 * (rows > 0)
    over = np.abs(got - value) - (half(dtype) * (1 + slack) * np.abs(value) + slack * (1 + half(dtype)) * mag + TINY)
    at = np.unravel_index(over.argmax(), over.shape)
    assert over.max() <= 0, f"{name}{at}: {got[at]!r} instead of {value[at]!r} (of {mag[at]!r})"


def make(rows, H, dtype, seed=0, y=True, gamma=True, beta=True, dh=True, mean=0.5):
    g = np.random.Generator(np.random.Philox(key=[seed + rows, H]))
    size = np.exp(0.5 * g.standard_normal((rows, 1)))
    rnd = lambda shape, std, at=0.0: rounded(std * (g.standard_normal(shape) + at), dtype)
    return dict(x=rnd((rows, H), 2 * size, mean), y=rnd((rows, H), 0.7 * size) if y else None,
                gamma=rnd(H, 0.2, 5.0) if gamma else None, beta=rnd(H, 0.3) if beta else None,
                h=rnd((rows, H), 2 * size, mean), dn=rnd((rows, H), 0.02), dh=rnd((rows, H), 0.01) if dh else None)


def vector(v, dtype):
    return None if v is None else torch.from_numpy(v).to(DT[dtype]).cuda()


def check_forward(rows, H, dtype, pad=0, front=0, eps=1e-5, in_place=False, **kw):
    import paper_2410_10989_amd as flce
    print(f"case forward {rows} {H} {dtype} {kw}", flush=True)
    c = make(rows, H, dtype, **kw)
    eps = float(np.float32(eps))
    ref = oracle.layer_norm(c["x"], c["y"], c["gamma"], c["beta"], eps)
    X = Matrix(rows, H, dtype, pad, front, c["x"])
    Y = Matrix(rows, H, dtype, pad, 0, c["y"]) if c["y"] is not None else None
    h = None if Y is None else X if in_place else Matrix(rows, H, dtype, pad, front)
    n = Matrix(rows, H, dtype, pad, 5)
    got = flce.flce_layer_norm_fwd(X.view, Y.view if Y else None, vector(c["gamma"], dtype), vector(c["beta"], dtype), eps,
                                   h=h.view if h else None, n=n.view)
    torch.cuda.synchronize()
    check("n", got[1], ref, dtype)
    n.assert_around_untouched()
    if Y:
        check("h", got[0], ref, dtype)
        h.assert_around_untouched()
    else:
        assert got[0] is None


SIZES = [(1, 1), (1, 64), (3, 7), (5, 8), (33, 9), (17, 127), (100, 128), (65, 130), (40, 512), (129, 513), (7, 1000), (9, 1024),
         (50, 1025), (4, 2048), (31, 2050), (6, 4095), (12, 4096), (5, 4097), (6, 8192), (3, 8200), (4, 12001), (2, 16384), (3, 16400),
         (2, 20001)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,H", SIZES)
def test_forward(rows, H, dtype):
    check_forward(rows, H, dtype)


@pytest.mark.parametrize("rows,H,dtype,kw", [
    (33, 520, "bf16", dict(y=False)), (33, 520, "f32", dict(gamma=False)), (33, 521, "bf16", dict(beta=False, pad=3, front=1)),
    (9, 4096, "bf16", dict(gamma=False, beta=False, pad=8)), (21, 1000, "f32", dict(pad=13, front=3, y=False, beta=False)),
    (16, 256, "f32", dict(mean=1000.0)), (16, 4096, "bf16", dict(mean=50.0, eps=0.0)), (5, 20000, "f32", dict(mean=100.0, pad=1)),
    (700, 96, "bf16", dict(in_place=True, pad=5)), (3, 17000, "bf16", dict(in_place=True)), (40, 8192, "f32", dict(in_place=True))])
def test_forward_variants(rows, H, dtype, kw):
    check_forward(rows, H, dtype, **kw)


def check_backward(rows, H, dtype, pad=0, front=0, eps=1e-5, in_place=False, workspace=None, flags=0, **kw):
    import paper_2410_10989_amd as flce
    print(f"case backward {rows} {H} {dtype} {kw}", flush=True)
    c = make(rows, H, dtype, **kw)
    eps = float(np.float32(eps))
    ref = oracle.layer_norm_grad(c["h"], c["dn"], c["dh"], c["gamma"], eps)
    put = lambda name, at=0: Matrix(rows, H, dtype, pad, at, c[name]) if c[name] is not None else None
    h, dn, dh = put("h", front), put("dn"), put("dh", 2)
    dx = dh if in_place else Matrix(rows, H, dtype, pad, front)
    vec = [Matrix(1, H, dtype, 0, 3) for _ in range(2)]
    has = c["gamma"] is not None
    got = flce.flce_layer_norm_bwd(h.view, dn.view, dh.view if dh else None, vector(c["gamma"], dtype), c["beta"] is not None, eps,
                                   dx=None if flags & flce.SKIP_DX else dx.view, dgamma=vec[0].view[0] if has and not flags & flce.SKIP_DW else None,
                                   dbeta=vec[1].view[0] if c["beta"] is not None and not flags & flce.SKIP_DW else None,
                                   workspace=workspace, flags=flags)
    torch.cuda.synchronize()
    assert [g is None for g in got] == [bool(flags & flce.SKIP_DX), not has or bool(flags & flce.SKIP_DW),
                                        c["beta"] is None or bool(flags & flce.SKIP_DW)]
    if got[0] is not None:
        check("dx", got[0], ref, dtype)
        dx.assert_around_untouched()
    for k, (name, m) in enumerate(zip(("dgamma", "dbeta"), vec)):
        if got[1 + k] is not None:
            check(name, got[1 + k], ref, dtype, rows)
            m.assert_around_untouched()
    return got


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,H", SIZES)
def test_backward(rows, H, dtype):
    check_backward(rows, H, dtype)


@pytest.mark.parametrize("rows,H,dtype,kw", [
    (2, 8, "f32", {}), (600, 24, "bf16", {}), (3000, 72, "f32", {}), (1025, 1000, "bf16", {}), (2049, 520, "f32", {}), (700, 2304, "bf16", {}),
    (33, 520, "bf16", dict(dh=False)), (33, 520, "f32", dict(gamma=False)), (33, 521, "bf16", dict(beta=False, pad=3, front=1)),
    (90, 4096, "bf16", dict(gamma=False, beta=False, pad=8)), (210, 1000, "f32", dict(pad=13, front=3, dh=False, beta=False)),
    (16, 256, "f32", dict(mean=1000.0)), (160, 4096, "bf16", dict(mean=50.0, eps=0.0)), (5, 20000, "f32", dict(mean=100.0, pad=1)),
    (700, 96, "bf16", dict(in_place=True, pad=5)), (3, 17000, "bf16", dict(in_place=True)), (400, 8192, "f32", dict(in_place=True)),
    (300, 12000, "bf16", {}), (50, 520, "f32", dict(flags=1)), (50, 520, "bf16", dict(flags=2)), (40, 5, "f32", dict(gamma=False, flags=1))])
def test_backward_variants(rows, H, dtype, kw):
    check_backward(rows, H, dtype, **kw)


@pytest.mark.parametrize("rows,H", [(3000, 136), (2000, 2304), (40, 20000)])
def test_smaller_workspaces_take_fewer_workgroups(rows, H):
    import paper_2410_10989_amd as flce
    full = flce.flce_layer_norm_workspace_bytes(rows, H, torch.float32)
    for n in {full, full // 3, 8 * H}:
        check_backward(rows, H, "f32", workspace=torch.full((n,), 255, dtype=torch.uint8, device="cuda"))
    short = torch.empty(4 * H - 4 if H == 20000 else 0, dtype=torch.uint8, device="cuda")
    if H == 20000:   # (the other shapes do with one workgroup, without partial sums)
        with pytest.raises(flce.FlceError) as e:
            check_backward(rows, H, "f32", workspace=short)
        assert e.value.status == 5


def test_gradient_against_differences_of_the_forward():
    """sum(n dn) + sum(h dh) of the library's own fp32 forward, changed along a direction by +-2^-6: the difference
    quotient is off by its second-order term (relative 2^-12 times a few) and by the forward's rounding, 2^-24 of about
    30 terms' magnitude over the step 2^-6, hence well below 2^-9 of the root of the sum of squares."""
    import paper_2410_10989_amd as flce
    g = torch.Generator(device="cuda").manual_seed(5)
    rows, H = 6, 40
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
    x, y, gamma, beta, dn, dh = rnd(rows, H), rnd(rows, H), rnd(H), rnd(H), rnd(rows, H), rnd(rows, H)

    def value(x, gamma, beta):
        h, n = flce.flce_layer_norm_fwd(x, y, gamma, beta, 1e-3)
        return ((h.double() * dh).sum() + (n.double() * dn).sum()).item()

    grads = flce.flce_layer_norm_bwd(x + y, dn, dh, gamma, True, 1e-3)
    for k, d in enumerate((rnd(rows, H), rnd(H), rnd(H))):
        step = [0.0, 0.0, 0.0]
        step[k] = 2.0 ** -6 * d
        up = value(x + step[0], gamma + step[1], beta + step[2])
        down = value(x - step[0], gamma - step[1], beta - step[2])
        along = (grads[k].double() * d).sum().item()
        scale = (grads[k].double() * d).square().sum().sqrt().item()
        assert abs((up - down) / 2.0 ** -5 - along) <= 2.0 ** -9 * max(scale, 1.0) * 4


def test_infinities_and_nan_stay_in_their_rows():
    import paper_2410_10989_amd as flce
    x = torch.randn(9, 72, device="cuda")
    want = flce.flce_layer_norm_fwd(x)[1]
    bad = x.clone()
    bad[2, 5], bad[4, 71], bad[7, 0] = float("inf"), float("nan"), -float("inf")
    got = flce.flce_layer_norm_fwd(bad)[1]
    hit = torch.tensor([2, 4, 7], device="cuda")
    rest = torch.tensor([0, 1, 3, 5, 6, 8], device="cuda")
    assert torch.equal(got[rest], want[rest]) and got[hit].isnan().any(1).all()


def test_rows_of_equal_elements():
    """d = 0: n is beta, and with eps the gradient stays finite (r = eps^-1/2)."""
    import paper_2410_10989_amd as flce
    x = torch.full((5, 33), 3.25, device="cuda")
    beta = torch.randn(33, device="cuda")
    assert torch.equal(flce.flce_layer_norm_fwd(x, beta=beta, gamma=beta)[1], beta.expand(5, 33))
    dx, dg, _ = flce.flce_layer_norm_bwd(x, torch.randn(5, 33, device="cuda"), gamma=beta)
    assert dx.isfinite().all() and (dg == 0).all()


def test_captured_calls_replay():
    import paper_2410_10989_amd as flce
    rows, H = 900, 264
    x, y, dn = (torch.randn(rows, H, device="cuda") for _ in range(3))
    gamma, beta = torch.randn(H, device="cuda"), torch.randn(H, device="cuda")
    h, n, dx = (torch.empty_like(x) for _ in range(3))
    dg, db = torch.empty_like(gamma), torch.empty_like(beta)

    def both():
        flce.flce_layer_norm_fwd(x, y, gamma, beta, h=h, n=n)
        flce.flce_layer_norm_bwd(h, dn, dn, gamma, dx=dx, dgamma=dg, dbeta=db)

    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for k in range(4):
        x.normal_()
        dn.normal_()
        graph.replay()
        torch.cuda.synchronize()
        hw, nw = flce.flce_layer_norm_fwd(x, y, gamma, beta)
        want = flce.flce_layer_norm_bwd(hw, dn, dn, gamma)
        assert all(torch.equal(a, b) for a, b in zip((h, n, dx, dg, db), (hw, nw, *want)))
        flce.flce_layer_norm_bwd(torch.randn(3000, 1000, device="cuda"), torch.randn(3000, 1000, device="cuda"))
