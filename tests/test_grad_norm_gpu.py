"""Global gradient norm and clipping against their 64-bit definition, through the binding.

Tolerances: the norm's squares are summed in fp64 (2^-53 each of at most 2^40 of them, far below the last
rounding): half a step of fp32.  The factor: that norm and the factor's own rounding, 2^-23; the product
rounds once more, to the storage type.
"""
import math

import numpy as np
import pytest
import torch

from oracle import block_norm_oracle as oracle

pytestmark = pytest.mark.gpu

NORM_TOL = 2.0 ** -24 * 1.001


def make(sizes, dtypes, seed, front=0, std=1.0):
    """Tensors as views of flat buffers, one element of mark between any two."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    bufs, views = [], []
    for i, n in enumerate(sizes):
        buf = torch.full((front + n + 1,), 77.0, dtype=dtypes[i % len(dtypes)], device="cuda")
        v = buf[front:front + n]
        v.copy_(torch.randn(n, generator=g, device="cuda") * (std * (1 + i % 3)))
        bufs.append(buf)
        views.append(v)
    return bufs, views


def host(ts):
    return [t.double().cpu().numpy() for t in ts]


def check_norm(got, ref):
    got = float(got)
    assert (math.isnan(ref) and math.isnan(got)) or got == ref or abs(got - ref) <= NORM_TOL * abs(ref), (got, ref)


def check_scaled(outs, ref, factor):
    for i, (o, r) in enumerate(zip(outs, ref)):
        half = torch.finfo(o.dtype).eps / 2
        o = o.double().cpu().numpy()
        want = r * factor
        assert np.all(np.abs(o - want) <= (half + 2.0 ** -22) * np.abs(want) + 2.0 ** -133), i


def clip(grads, norm_type, ratio, outs=None):
    import paper_2410_10989_amd as flce
    ref = host(grads)
    kind = "2" if norm_type == 2.0 else "inf"
    norm = oracle.grad_norm(ref, kind)
    most = ratio * norm if norm > 0 and math.isfinite(norm) else 1.0
    check_norm(flce.flce_grad_norm(grads, norm_type), norm)
    got = flce.flce_clip_grad_norm(grads, most, norm_type, outs=outs)
    torch.cuda.synchronize()
    check_norm(got, norm)
    check_scaled(outs if outs is not None else grads, ref, oracle.clip_factor(norm, most))


F, B = torch.float32, torch.bfloat16
LISTS = [([1], [F]), ([1], [B]), ([7, 0, 9], [B, F]), ([0, 0], [F]), ([255, 256, 257, 4095, 4097], [F]),
         ([8191, 8193, 65537, 3], [B]), ([1 << 20, (1 << 20) + 5], [B, F]), ([3 + 17 * i % 1000 for i in range(120)], [B, F]),
         ([1 + 31 * i % 700 for i in range(121)], [F, B]), ([i % 50 for i in range(700)], [B]),
         ([5_000_011, 10, 3_000_003], [F, B, F])]


@pytest.mark.parametrize("front", [0, 1, 3])
@pytest.mark.parametrize("norm_type", [2.0, math.inf])
@pytest.mark.parametrize("sizes,dtypes", LISTS, ids=lambda v: f"{len(v)}")
def test_norm_and_clip(sizes, dtypes, norm_type, front):
    print(f"case clip {len(sizes)} tensors of {sum(sizes)}, {dtypes}, {norm_type}, front {front}", flush=True)
    for ratio in (0.3, 1.7):
        bufs, grads = make(sizes, dtypes, 1 + len(sizes), front)
        outs_bufs, outs = make(sizes, dtypes, 2, front + 1)
        before = [g.clone() for g in grads]
        clip(grads, norm_type, ratio, outs=outs)
        assert all(torch.equal(a, b) for a, b in zip(before, grads)), "inputs changed"
        clip(grads, norm_type, ratio)
        for b, f in [(b, front) for b in bufs] + [(b, front + 1) for b in outs_bufs]:
            assert (b[:f] == 77).all() and (b[-1:] == 77).all(), "written outside a tensor"


@pytest.mark.parametrize("norm_type", [2.0, math.inf])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_a_norm_that_is_not_finite_scales_nothing(value, norm_type):
    import paper_2410_10989_amd as flce
    for where in (0, 70_000, 131_071):
        _, grads = make([131_072, 77], [F, B], 3)
        grads[0][where] = value
        before = [g.clone() for g in grads]
        outs = [torch.empty_like(g) for g in grads]
        norm = flce.flce_clip_grad_norm(grads, 0.5, norm_type, outs=outs)
        assert math.isnan(norm) if math.isnan(value) else math.isinf(norm)
        flce.flce_clip_grad_norm(grads, 0.5, norm_type)
        for a, b, c in zip(before, grads, outs):
            assert torch.equal(a.view(torch.int16), b.view(torch.int16)) and torch.equal(a.view(torch.int16), c.view(torch.int16))


def test_values_whose_squares_leave_the_range_of_fp32():
    for std in (1e30, 1e-30):
        _, grads = make([5000, 333], [F, B], 4, std=std)
        clip(grads, 2.0, 0.5, outs=[torch.empty_like(g) for g in grads])


def test_the_smallest_numbers_are_kept():
    """Numbers below the normal range of fp32 and bf16, scaled by 1 and by 1/2."""
    import paper_2410_10989_amd as flce
    t = [torch.full((300,), 2.0 ** -140, device="cuda"), torch.full((70,), 2.0 ** -130, dtype=torch.bfloat16, device="cuda")]
    norm = torch.ones((), device="cuda")
    outs = [torch.zeros_like(v) for v in t]
    flce.flce_grad_clip(t, norm, 2.0, outs=outs)
    assert all(torch.equal(a, b) for a, b in zip(outs, t))
    flce.flce_grad_clip(t, norm * (2.0 - 1e-6), 1.0, outs=outs)
    assert (outs[0] == 2.0 ** -141).all() and (outs[1] == 2.0 ** -131).all()


def test_zero_gradients_and_a_threshold_of_zero():
    import paper_2410_10989_amd as flce
    z = [torch.zeros(1000, device="cuda"), torch.zeros(3, dtype=B, device="cuda")]
    assert float(flce.flce_clip_grad_norm(z, 1.0)) == 0 and not any(t.any() for t in z)
    _, grads = make([1000], [F], 5)
    assert float(flce.flce_clip_grad_norm(grads, 0.0)) > 0 and not grads[0].any()
    norm = torch.full((), 5.0, device="cuda")
    assert flce.flce_clip_grad_norm([], 1.0, norm=norm) is norm and float(norm) == 0
    norm.fill_(5.0)
    assert float(flce.flce_grad_norm([], norm=norm)) == 0


def test_a_norm_of_several_shards():
    import paper_2410_10989_amd as flce
    _, grads = make([4097, 12, 30_001], [F, B], 6)
    ref = host(grads)
    whole = flce.flce_grad_norm(grads)
    parts = torch.stack([flce.flce_grad_norm(grads[:1]), flce.flce_grad_norm(grads[1:])])
    total = parts.square().sum().sqrt()
    flce.flce_grad_clip(grads, total, 2.0)
    check_scaled(grads, ref, oracle.clip_factor(float(total), 2.0))
    assert abs(float(total) - float(whole)) <= 4 * 2.0 ** -24 * float(whole)


def test_same_bits_on_another_stream_and_with_a_workspace_of_its_own():
    import paper_2410_10989_amd as flce
    _, grads = make([100_003, 70_000, 5] * 60, [B, F], 7)
    outs = [torch.empty_like(g) for g in grads]
    want = flce.flce_clip_grad_norm(grads, 1.0, outs=outs)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    need = flce.flce_grad_norm_workspace_bytes(len(grads))
    ws = torch.full((need + 256,), 255, dtype=torch.uint8, device="cuda")
    for _ in range(3):
        outs2 = [torch.empty_like(g) for g in grads]
        torch.cuda.synchronize()
        got = flce.flce_clip_grad_norm(grads, 1.0, outs=outs2, workspace=ws[:need], stream=side)
        side.synchronize()
        assert float(got) == float(want) and all(torch.equal(a, b) for a, b in zip(outs, outs2))
        assert (ws[need:] == 255).all()


def test_captured_and_replayed():
    import paper_2410_10989_amd as flce
    _, grads = make([50_001, 333, 8] * 50, [F, B], 8)
    ws = torch.empty(flce.flce_grad_norm_workspace_bytes(len(grads)), dtype=torch.uint8, device="cuda")
    norm = torch.empty((), device="cuda")
    outs = [torch.empty_like(g) for g in grads]
    flce.flce_clip_grad_norm(grads, 1.0, outs=outs, norm=norm, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        flce.flce_clip_grad_norm(grads, 1.0, outs=outs, norm=norm, workspace=ws)
    for turn in range(4):
        for g in grads:
            g.mul_(1.5)
        for o in outs:
            o.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        mine = [torch.empty_like(g) for g in grads]
        want = flce.flce_clip_grad_norm(grads, 1.0, outs=mine)
        assert float(norm) == float(want) and all(torch.equal(a, b) for a, b in zip(outs, mine)), turn


def test_a_short_list_is_captured_where_the_library_has_no_workspace():
    import paper_2410_10989_amd as flce
    _, grads = make([4000, 77, 0, 1], [F, B], 9)
    norm = torch.empty((), device="cuda")
    outs = [torch.empty_like(g) for g in grads]
    assert flce.lib().flce_release_workspace() == 0
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        flce.flce_clip_grad_norm(grads, 1.0, outs=outs, norm=norm)
    for turn in range(3):
        for g in grads:
            g.mul_(1.5)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        ref = host(grads)
        check_norm(norm, oracle.grad_norm(ref))
        check_scaled(outs, ref, oracle.clip_factor(oracle.grad_norm(ref), 1.0))


def test_a_tensor_of_more_than_2_to_the_31_elements():
    import paper_2410_10989_amd as flce
    n = (1 << 31) + 77
    g = torch.empty(n, dtype=B, device="cuda").fill_(0.5)
    g[-1] = 3.0
    norm = flce.flce_clip_grad_norm([g], 1.0)
    check_norm(norm, math.sqrt(0.25 * (n - 1) + 9.0))
    f = 1.0 / (float(norm) + 1e-6)
    for at in (0, 1, (1 << 31) - 1, 1 << 31, n - 2):
        assert abs(float(g[at]) - 0.5 * f) <= (2.0 ** -8 + 2.0 ** -22) * 0.5 * f
    assert abs(float(g[-1]) - 3 * f) <= (2.0 ** -8 + 2.0 ** -22) * 3 * f
    assert float(g[:1 << 30].max()) == float(g[:1 << 30].min()) == float(g[(1 << 31) - 9:-1].min())


def test_binding_refusals():
    import paper_2410_10989_amd as flce
    g = torch.ones(4, 6, device="cuda")
    for bad in ([g, g.cpu()], [g.t()], [g.half()]):
        with pytest.raises((ValueError, TypeError)):
            flce.flce_grad_norm(bad)
    for kw in (dict(norm_type=1.0), dict(outs=[]), dict(outs=[g.bfloat16()]), dict(outs=[g[:2].clone()]),
               dict(norm=torch.zeros((), dtype=torch.float64, device="cuda"))):
        with pytest.raises((ValueError, KeyError)):
            flce.flce_clip_grad_norm([g], 1.0, **kw)
    with pytest.raises(ValueError):
        flce.flce_grad_norm([g], workspace=torch.empty(1 << 20, dtype=torch.uint8))
    for grads in ([g, g], [g, g[1:3]]):
        with pytest.raises(flce.FlceError) as e:
            flce.flce_clip_grad_norm(grads, 1.0)
        assert e.value.status == 7
    with pytest.raises(flce.FlceError) as e:
        flce.flce_clip_grad_norm([g], -1.0)
    assert e.value.status == 7 and (g == 1).all()
