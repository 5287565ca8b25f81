"""Newton-Schulz orthogonalisation against its 64-bit definition.

Tolerances.  The iteration amplifies roundings by factors that depend on the matrix, so each case's error is measured
against what the roundings that the header names do by themselves: the 64-bit definition with fp16 planes and fp32 sums
(oracle.orthogonalize_rounded) is off by some amount; the kernels make the same roundings of values that differ in
their last bits (other orders of the fp32 sums), i.e. another sample of the same error, and may be off twice as far
in the 2-norm, four times in the largest element (the maximum of another sample), plus half a step of the output's
type, plus 2^-21 of the norm (a floor for the fp32 sums of tiny matrices, whose two samples may be lucky).
"""
import numpy as np
import pytest
import torch

from matrices import DT, half, rounded
from oracle import step_oracle as oracle

pytestmark = pytest.mark.gpu


def make(rows, cols, dtype, seed=0, rank=3, spike=1.0):
    g = np.random.Generator(np.random.Philox(key=[rows + seed, cols]))
    G = g.standard_normal((rows, cols))
    if rank:
        G = G + spike * g.standard_normal((rows, rank)) @ g.standard_normal((rank, cols)) / np.sqrt(rank)
    return rounded(1e-3 * G, dtype)


def check(got, G, dtype, **kw):
    ref = oracle.orthogonalize(G, **kw)
    model = oracle.orthogonalize_rounded(G, 2 if dtype == "f32" else 1, **kw)
    got = got.double().cpu().numpy()
    assert got.shape == ref.shape and np.isfinite(got).all()
    off, may = np.linalg.norm(got - ref), 2 * np.linalg.norm(model - ref) + (half(dtype) + 2.0 ** -21) * np.linalg.norm(ref)
    worst = np.abs(got - ref).max()
    may_worst = 4 * np.abs(model - ref).max() + (half(dtype) + 2.0 ** -21) * np.abs(ref).max()
    print(f"off {off / np.linalg.norm(ref):.2e}, may be {may / np.linalg.norm(ref):.2e}", flush=True)
    assert off <= may and worst <= may_worst


SHAPES = [(1, 1), (1, 9), (7, 1), (3, 5), (16, 16), (64, 64), (65, 64), (63, 200), (200, 63), (128, 128), (129, 127), (100, 1000), (1000, 100),
          (256, 256), (257, 300), (16, 4099), (520, 260), (512, 512)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_one_matrix(rows, cols, dtype):
    import paper_2410_10989_amd as flce
    print(f"case {rows} {cols} {dtype}", flush=True)
    G = make(rows, cols, dtype)
    t = torch.from_numpy(G).to(DT[dtype]).cuda()
    out = torch.full((rows * cols + 16,), 77.0, dtype=DT[dtype], device="cuda")
    view = out[8:8 + rows * cols].view(rows, cols).fill_(float("nan"))
    got = flce.flce_orthogonalize([t], outs=[view])
    torch.cuda.synchronize()
    assert got[0] is view
    check(view, G, dtype)
    assert (out[:8] == 77.0).all() and (out[8 + rows * cols:] == 77.0).all()
    assert torch.equal(t.double().cpu(), torch.from_numpy(G))
    flce.flce_orthogonalize([t])   # in place
    assert torch.equal(t, view)


@pytest.mark.parametrize("dtype,count,rows,cols", [("bf16", 5, 130, 70), ("f32", 3, 70, 130), ("bf16", 130, 33, 40), ("bf16", 20, 512, 512),
                                                   ("f32", 14, 512, 768), ("bf16", 9, 1025, 600), ("bf16", 50, 300, 640),
                                                   ("bf16", 45, 1300, 520), ("f32", 44, 384, 800), ("f32", 50, 777, 323), ("f32", 90, 300, 640)])
def test_lists(dtype, count, rows, cols):
    """Many matrices of a list, on both sizes of tiles, in several groups of launches."""
    import paper_2410_10989_amd as flce
    print(f"case list of {count} {rows} {cols} {dtype}", flush=True)
    G = [make(rows, cols, dtype, seed=i % 4) for i in range(4)]
    ts = [torch.from_numpy(G[i % 4]).to(DT[dtype]).cuda() for i in range(count)]
    outs = [torch.empty_like(t) for t in ts]
    flce.flce_orthogonalize(ts, outs=outs, scale=0.3)
    torch.cuda.synchronize()
    for i in range(min(4, count)):
        check(outs[i], G[i], dtype, scale=float(np.float32(0.3)))
    assert all(torch.equal(o, outs[i % 4]) for i, o in enumerate(outs))


@pytest.mark.parametrize("kw", [dict(steps=1), dict(steps=3, coefficients=(2.0, -1.5, 0.5)), dict(steps=4, coefficients=(1.5, -0.5, 0.0)),
                                dict(steps=2, coefficients=[(8.0, -22.0, 16.0), (4.0, -3.0, 0.5)]), dict(steps=1, coefficients=(0.0, 1.0, 0.0)),
                                dict(scale=-7.0), dict(eps=0.5), dict(steps=8)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_other_polynomials(kw, dtype):
    import paper_2410_10989_amd as flce
    G = make(90, 140, dtype)
    got = flce.flce_orthogonalize([torch.from_numpy(G).to(DT[dtype]).cuda()], **kw)[0]
    torch.cuda.synchronize()
    check(got, G, dtype, **{k: float(np.float32(v)) if k == "eps" else v for k, v in kw.items()})


@pytest.mark.parametrize("rows,cols,count", [(700, 400, 1), (400, 700, 1), (301, 450, 50), (450, 301, 50)])
def test_last_step_that_multiplies_errors(rows, cols, count):
    """The last product adds X's second plane, of columns where the matrix is tall."""
    import paper_2410_10989_amd as flce
    G = make(rows, cols, "bf16")
    kw = dict(steps=2, coefficients=[(3.4445, -4.775, 2.0315), (20.0, -30.0, 11.0)])
    got = flce.flce_orthogonalize([torch.from_numpy(G).bfloat16().cuda() for _ in range(count)], **kw)
    check(got[-1], G, "bf16", **{**kw, "coefficients": np.float32(kw["coefficients"]).astype(float).tolist()})
    assert torch.equal(got[0], got[-1])


@pytest.mark.parametrize("dtype,rows,cols,count", [("f32", 192, 192, 1), ("bf16", 192, 192, 1), ("bf16", 60, 100, 1), ("bf16", 128, 128, 1),
                                                   ("bf16", 320, 320, 1), ("bf16", 300, 700, 50), ("f32", 300, 700, 50)])
def test_matrices_of_low_rank(dtype, rows, cols, count):
    """A gradient of rank 2 and a little noise: X is carried over in more than 11 bits."""
    import paper_2410_10989_amd as flce
    G = make(rows, cols, dtype, rank=2, spike=30.0)
    got = flce.flce_orthogonalize([torch.from_numpy(G).to(DT[dtype]).cuda() for _ in range(count)])[-1]
    check(got, G, dtype)
    ref = oracle.orthogonalize(G)
    assert np.linalg.norm(got.double().cpu().numpy() - ref) <= (5e-3 if dtype == "bf16" else 1e-4) * np.linalg.norm(ref)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [2.0 ** -120, 2.0 ** -60, 2.0 ** 60, 2.0 ** 120])
def test_sizes_of_the_elements(dtype, size):
    """Squares are summed in fp64: they neither overflow nor vanish."""
    import paper_2410_10989_amd as flce
    G = size * make(40, 60, dtype) * 1e3
    got = flce.flce_orthogonalize([torch.from_numpy(G).to(DT[dtype]).cuda()], eps=0.0)[0]
    check(got, G, dtype, eps=0.0)


def test_zeros_infinities_and_nan():
    import paper_2410_10989_amd as flce
    ts = [torch.randn(70, 90, device="cuda") for _ in range(5)]
    want = [t.clone() for t in ts]
    flce.flce_orthogonalize(want)
    ts[1].zero_()
    ts[2][3, 4] = float("inf")
    ts[3][69, 89] = float("nan")
    flce.flce_orthogonalize(ts)
    assert torch.equal(ts[0], want[0]) and torch.equal(ts[4], want[4])
    assert (ts[1] == 0).all() and ts[2].isnan().all() and ts[3].isnan().all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(37, 90), (90, 37), (300, 261), (261, 300)])
def test_matrices_at_any_element(rows, cols, dtype):
    """Neither matrix nor result begins on 16 bytes, nor do their rows; what lies around the result stays."""
    import paper_2410_10989_amd as flce
    G = make(rows, cols, dtype)
    n = rows * cols
    room = torch.zeros(n + 16, dtype=DT[dtype], device="cuda")
    to = torch.full((n + 16,), 77.0, dtype=DT[dtype], device="cuda")
    t, out = room[1:1 + n].view(rows, cols), to[3:3 + n].view(rows, cols)
    t.copy_(torch.from_numpy(G))
    flce.flce_orthogonalize([t], outs=[out])
    check(out, G, dtype)
    assert (to[:3] == 77.0).all() and (to[3 + n:] == 77.0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_zeros_without_eps(dtype):
    import paper_2410_10989_amd as flce
    for shape in ((5, 9), (300, 200)):
        ts = [torch.zeros(shape, dtype=DT[dtype], device="cuda") for _ in range(2)]
        ts[1][2, 3] = 4.0
        got = flce.flce_orthogonalize(ts, outs=[torch.empty_like(t) for t in ts], eps=0.0)
        assert (got[0] == 0).all()
        check(got[1], ts[1].double().cpu().numpy(), dtype, eps=0.0)


def test_a_matrix_that_is_read_twice():
    """The same update under two results, and in place among others."""
    import paper_2410_10989_amd as flce
    a, b = (torch.randn(80, 70, device="cuda") for _ in range(2))
    want = flce.flce_orthogonalize([a, b], outs=[torch.empty_like(a) for _ in range(2)])
    outs = [torch.empty_like(a), torch.empty_like(a), b]
    flce.flce_orthogonalize([a, a, b], outs=outs)
    assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[0]) and torch.equal(b, want[1])
    with pytest.raises(flce.FlceError):
        flce.flce_orthogonalize([a, a])
    with pytest.raises(flce.FlceError):
        flce.flce_orthogonalize([a, b], outs=[torch.empty_like(a), a])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_smaller_workspaces_take_fewer_matrices_at_a_time(dtype):
    import paper_2410_10989_amd as flce
    G = [make(140, 90, dtype, seed=i) for i in range(6)]
    ts = [torch.from_numpy(g).to(DT[dtype]).cuda() for g in G]
    one = flce.flce_orthogonalize_workspace_bytes(1, 140, 90, DT[dtype])
    for n in (6 * one, 4 * one + 100, one):
        ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
        outs = flce.flce_orthogonalize(ts, outs=[torch.empty_like(t) for t in ts], workspace=ws)
        for o, g in zip(outs, G):
            check(o, g, dtype)
    with pytest.raises(flce.FlceError) as e:
        flce.flce_orthogonalize(ts, workspace=torch.empty(one - 1, dtype=torch.uint8, device="cuda"))
    assert e.value.status == 5


def test_captured_calls_replay():
    import paper_2410_10989_amd as flce
    ts = [torch.randn(100, 300, device="cuda").bfloat16() for _ in range(3)]
    outs = [torch.empty_like(t) for t in ts]
    flce.flce_orthogonalize(ts, outs=outs)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        flce.flce_orthogonalize(ts, outs=outs)
    for _ in range(4):
        for t in ts:
            t.normal_()
        graph.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in outs]
        want = flce.flce_orthogonalize(ts, outs=[torch.empty_like(t) for t in ts])
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        flce.flce_orthogonalize([torch.randn(400, 500, device="cuda")])


def test_calls_on_two_streams_with_their_own_workspaces():
    import paper_2410_10989_amd as flce
    ts = [torch.randn(300, 200, device="cuda") for _ in range(2)]
    want = flce.flce_orthogonalize(ts, outs=[torch.empty_like(t) for t in ts])
    n = flce.flce_orthogonalize_workspace_bytes(1, 300, 200, torch.float32)
    ws = [torch.empty(n, dtype=torch.uint8, device="cuda") for _ in ts]
    got = [torch.empty_like(t) for t in ts]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in ts]
    for _ in range(3):
        for t, o, w, s in zip(ts, got, ws, streams):
            flce.flce_orthogonalize([t], outs=[o], workspace=w, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
