"""Norms around a block (forward and backward) against their 64-bit definition, through the binding.

Tolerances, element by element: half a step of the storage type of the value (one rounding of the output), plus
2^-17 of the magnitude of what was added up to it.  The latter covers fp32 arithmetic: a row's sum of squares
(at most 16 terms one after the other per thread, or H / 1024 in the long form, then a tree) is off by less than
(16 + H / 1024 + 16) 2^-24 <= 2^-18 for H <= 32768, which a square root halves; up to a dozen factors of 2^-24
each; a(g), a'(g) to 2^-21.  Sums over rows: one more 2^-24 of the terms' magnitudes per row and partial sum.
"""
import numpy as np
import pytest
import torch

from oracle import block_norm_oracle as oracle

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
ARITH = 2.0 ** -17
TINY = 2.0 ** -126   # results below the normal range


def _tol(value, mag, dtype, rows=0, arith=ARITH):
    half = torch.finfo(DT[dtype]).eps / 2
    slack = arith + (rows + 32) * 2.0 ** -24 * (rows > 0)
    return (half * (1 + slack)) * np.abs(value) + slack * (1 + half) * mag + TINY


def _check(name, got, ref, dtype, rows=0, arith=ARITH):
    value, mag = ref[name], ref[name + "_mag"]
    got = got.double().cpu().numpy()
    assert got.shape == value.shape, name
    assert np.isfinite(got).all(), f"{name}: not finite"
    over = np.abs(got - value) - _tol(value, mag, dtype, rows, arith)
    at = np.unravel_index(over.argmax(), over.shape)
    assert over.max() <= 0, f"{name}{at}: {got[at]!r} instead of {value[at]!r} (of {mag[at]!r})"


class Matrix:
    """A [rows, H] matrix inside a wider buffer: `front` elements in front of it, rows `pad` elements longer,
    everything around it filled with a mark."""
    MARK = 77.0

    def __init__(self, rows, H, dtype, pad=0, front=0, data=None):
        self.buf = torch.full((front + rows * (H + pad) + 3,), self.MARK, dtype=DT[dtype], device="cuda")
        self.view = self.buf[front:front + rows * (H + pad)].view(rows, H + pad)[:, :H]
        if data is None:
            self.view.fill_(float("nan"))   # outputs must be overwritten
        else:
            self.view.copy_(torch.from_numpy(data))

    def assert_around_untouched(self):
        inside = self.view.clone()
        self.view.fill_(self.MARK)
        assert (self.buf == self.MARK).all(), "written outside the rows"
        self.view.copy_(inside)


def make(rows, H, dtype, seed, x=True, y=True, pre=True, post=False, gate="none", kind="linear", per=0, scale=0.75,
         eps=1e-6, pad=0, front=0):
    g = np.random.Generator(np.random.Philox(key=[seed, 31]))
    rnd = lambda shape, std=1.0, mean=0.0: torch.from_numpy(g.standard_normal(shape) * std + mean).to(DT[dtype]).double().numpy()
    size = np.exp(0.5 * g.standard_normal((rows, 1)))
    per = {"none": 0, "channel": 0, "token": 1}.get(gate, per)
    gshape = (H,) if per == 0 else (-(-rows // per), H)
    c = dict(rows=rows, H=H, dtype=dtype, pad=pad, front=front,
             x=rnd((rows, H), 2.0 * size) if x else None, y=rnd((rows, H), 0.7 * size) if y else None,
             gate=rnd(gshape, 1.5) if gate != "none" else None, gamma_post=rnd(H, 0.2, 1.0) if post else None,
             gamma_pre=rnd(H, 0.2, 1.0) if pre else None, dn=rnd((rows, H), 0.02) if pre else None,
             dh=rnd((rows, H), 0.01) if x or not pre else None, h=rnd((rows, H), 1.5 * size) if pre else None,
             opt=dict(kind=kind, rows_per_gate=per, scale=float(np.float32(scale)), eps=float(np.float32(eps))))
    return c


def _dev(c, name):
    v = c[name]
    if v is None:
        return None
    return Matrix(*v.shape, c["dtype"], c["pad"], c["front"], v).view if v.ndim == 2 else torch.from_numpy(v).to(DT[c["dtype"]]).cuda()


def _kw(c):
    o = c["opt"]
    return dict(gamma_pre=_dev(c, "gamma_pre"), gamma_post=_dev(c, "gamma_post"), gate=_dev(c, "gate"), gate_act=o["kind"],
                rows_per_gate=o["rows_per_gate"], scale=o["scale"], eps=o["eps"])


def check_forward(c):
    import paper_2410_10989_amd as flce
    ref = oracle.forward(c["x"], c["y"], c["gate"], c["gamma_post"], c["gamma_pre"], **c["opt"])
    outs = {k: Matrix(c["rows"], c["H"], c["dtype"], c["pad"], c["front"]) for k in ("h", "n") if k in ref}
    given = {k: m.view for k, m in outs.items()}
    h, n = flce.flce_block_norm_fwd(_dev(c, "x"), _dev(c, "y"), **_kw(c), **given)
    torch.cuda.synchronize()
    assert h is given.get("h") and n is given.get("n")
    for k, m in outs.items():
        _check(k, m.view, ref, c["dtype"])
        m.assert_around_untouched()


def reference_backward(c):
    return oracle.backward(c["h"], c["dn"], c["dh"], c["y"], c["gate"], c["gamma_post"], c["gamma_pre"], **c["opt"])


def rows_summed(c, name):
    per = c["opt"]["rows_per_gate"]
    if name in ("dx", "dy") or (name == "dgate" and per == 1):
        return 0
    return c["rows"] if name != "dgate" or per == 0 else min(c["rows"], per)


def check_backward(c, **kw):
    import paper_2410_10989_amd as flce
    ref = reference_backward(c)
    outs = {}
    for k in ("dx", "dy", "dgate"):
        if k in ref:
            shape = ref[k].shape if ref[k].ndim == 2 else (1,) + ref[k].shape
            outs[k] = Matrix(*shape, c["dtype"], c["pad"], c["front"])
    given = {k: m.view if ref[k].ndim == 2 else m.view[0] for k, m in outs.items()}
    got = flce.flce_block_norm_bwd(_dev(c, "h"), _dev(c, "dn"), _dev(c, "dh"), _dev(c, "y"), **_kw(c), **given, **kw)
    torch.cuda.synchronize()
    for name, t in zip(("dx", "dy", "dgate", "dgamma_post", "dgamma_pre"), got):
        assert (t is None) == (name not in ref), name
        if t is not None:
            _check(name, t, ref, c["dtype"], rows_summed(c, name))
    for m in outs.values():
        m.assert_around_untouched()


# the edges of the kernels' shapes: 16 .. 1024 threads per row, vectors that end inside a row, the long form
WIDTHS = [1, 3, 8, 9, 100, 127, 128, 129, 500, 512, 520, 1000, 1025, 2048, 2051, 2304, 4095, 4096, 4100, 8192, 8195, 13312, 13320, 16384, 16392, 20001]
VARIANTS = [dict(), dict(post=True), dict(gate="channel", kind="sigmoid"), dict(post=True, gate="channel", kind="linear"),
            dict(post=True, gate="sequence", per=5, kind="silu"), dict(gate="sequence", per=2, kind="tanh"),
            dict(post=True, gate="token", kind="tanh"), dict(gate="token", kind="silu"), dict(y=False),
            dict(x=False, post=True), dict(pre=False, post=True, gate="channel", kind="silu"), dict(x=False, gate="token", kind="sigmoid")]


def _widths():
    out = []
    for i, H in enumerate(WIDTHS):
        rows = [1, 2, 5, 19, 37][i % 5] if H > 2000 else [1, 33, 67, 18][i % 4]
        for j in range(4):
            v = VARIANTS[(3 * i + 5 * j) % len(VARIANTS)]
            out.append((rows, H, ("bf16", "f32")[(i + j) % 2], v, (i + j) % 3 and 5 * j, (i + 2 * j) % 4))
    return out


def _name(v):
    return "-".join(f"{k}={w}" for k, w in v.items()) or "plain" if isinstance(v, dict) else None


@pytest.mark.parametrize("rows,H,dtype,variant,pad,front", _widths(), ids=_name)
def test_forward_at_every_width(rows, H, dtype, variant, pad, front):
    print(f"case forward rows={rows} H={H} {dtype} {variant} pad={pad} front={front}", flush=True)
    check_forward(make(rows, H, dtype, 100 + H, pad=pad, front=front, **variant))


@pytest.mark.parametrize("rows,H,dtype,variant,pad,front", _widths(), ids=_name)
def test_backward_at_every_width(rows, H, dtype, variant, pad, front):
    print(f"case backward rows={rows} H={H} {dtype} {variant} pad={pad} front={front}", flush=True)
    check_backward(make(rows, H, dtype, 200 + H, pad=pad, front=front, **variant))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("variant", VARIANTS, ids=_name)
def test_every_variant(variant, dtype):
    print(f"case variant {variant} {dtype}", flush=True)
    for rows, H in ((50, 264), (23, 1100)):
        check_forward(make(rows, H, dtype, 5, **variant))
        check_backward(make(rows, H, dtype, 6, **variant))


@pytest.mark.parametrize("rows,H,dtype,variant", [
    (2500, 128, "bf16", dict(post=True, gate="channel", kind="silu")),       # more rows than groups of 16 threads
    (5000, 64, "f32", dict(gate="sequence", per=7, kind="sigmoid")),         # more gate rows than workgroups can cut
    (1500, 520, "bf16", dict(post=True, gate="sequence", per=400, kind="tanh")),   # gate rows cut into parts
    (1301, 2048, "bf16", dict(post=True)), (2600, 1024, "f32", dict(gate="token", kind="linear")),
    (1111, 4096, "bf16", dict(gate="sequence", per=1200, kind="silu")),      # one gate row, not quite used up
    (700, 8200, "bf16", dict(post=True, gate="sequence", per=100)),          # sums in LDS, several rows per workgroup
    (600, 8200, "f32", dict(gate="sequence", per=2, kind="tanh")),           # ... and more gate rows than workgroups
    (500, 13400, "bf16", dict(post=True, gate="sequence", per=100)),         # long form: three sets beyond the LDS
    (300, 16500, "f32", dict(gate="sequence", per=1, kind="tanh")), (520, 16500, "bf16", dict(gate="sequence", per=2)),
], ids=_name)
def test_many_rows(rows, H, dtype, variant):
    print(f"case many rows={rows} H={H} {dtype} {variant}", flush=True)
    check_forward(make(rows, H, dtype, 7, **variant))
    check_backward(make(rows, H, dtype, 8, **variant))


@pytest.mark.parametrize("rows,H", [(2, 4096), (3, 4096), (4, 4096), (12, 1000), (13, 1000), (48, 100), (49, 100), (3, 9000), (2, 20000)])
@pytest.mark.parametrize("variant", [dict(post=True, gate="channel", kind="tanh"), dict(post=True, gate="sequence", per=2),
                                     dict(gate="token", kind="silu")], ids=_name)
def test_a_handful_of_rows(rows, H, variant):
    """On both sides of where one workgroup takes all rows."""
    for dtype in ("bf16", "f32"):
        check_backward(make(rows, H, dtype, 25, **variant))


@pytest.mark.parametrize("shape", [(300, 1024), (40, 4096), (9, 16400)])
def test_a_smaller_workspace_serves(shape):
    """Fewer workgroups, down to one: 12 H bytes."""
    rows, H = shape
    for nbytes in (12 * H, 40 * H):
        ws = torch.full((nbytes // 4 + 64,), float("nan"), dtype=torch.float32, device="cuda")
        check_backward(make(rows, H, "bf16", 9, post=True, gate="channel", kind="sigmoid"), workspace=ws[:nbytes // 4])
        assert torch.isnan(ws[nbytes // 4:]).all(), "written past the workspace"


def test_h_may_lie_on_x_and_dx_on_dh():
    import paper_2410_10989_amd as flce
    for H in (96, 2304, 20000):
        c = make(21, H, "bf16", 10, post=True)
        x, y = _dev(c, "x"), _dev(c, "y")
        h, n = flce.flce_block_norm_fwd(x, y, **_kw(c))
        h2, n2 = flce.flce_block_norm_fwd(x, y, **_kw(c), h=x)
        assert h2 is x and torch.equal(h, h2) and torch.equal(n, n2)
        dn, dh = _dev(c, "dn"), _dev(c, "dh")
        a = flce.flce_block_norm_bwd(h, dn, dh, y, **_kw(c))
        b = flce.flce_block_norm_bwd(h, dn, dh, y, **_kw(c), dx=dh)
        assert b[0] is dh and all(torch.equal(u, v) for u, v in zip(a, b) if u is not None)


def test_h_on_x_that_is_y_and_the_gate_too():
    import paper_2410_10989_amd as flce
    for H in (96, 2304, 20000):
        c = make(21, H, "bf16", 27, post=True)
        x = _dev(c, "x")
        kw = dict(_kw(c), gate=x, gate_act="sigmoid", rows_per_gate=1)
        h, n = flce.flce_block_norm_fwd(x, x, **kw)
        h2, n2 = flce.flce_block_norm_fwd(x, x, **kw, h=x)
        assert h2 is x and torch.equal(h, h2) and torch.equal(n, n2)


def test_outputs_as_columns_of_one_wider_buffer():
    import paper_2410_10989_amd as flce
    c = make(31, 200, "f32", 11, post=True)
    kw = _kw(c)
    x, y, h, dn, dh = (_dev(c, k) for k in ("x", "y", "h", "dn", "dh"))
    want = flce.flce_block_norm_bwd(h, dn, dh, y, **kw)
    both = torch.empty(31, 401, device="cuda")
    got = flce.flce_block_norm_bwd(h, dn, dh, y, **kw, dx=both[:, :200], dy=both[:, 201:])
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    with pytest.raises(flce.FlceError) as e:
        flce.flce_block_norm_bwd(h, dn, dh, y, **kw, dx=both[:, :200], dy=both[:, 199:399])
    assert e.value.status == 7


def test_frozen_sides_and_missing_parts():
    import paper_2410_10989_amd as flce
    c = make(40, 300, "bf16", 12, post=True, gate="channel")
    kw, t = _kw(c), {k: _dev(c, k) for k in ("h", "dn", "dh", "y")}
    full = flce.flce_block_norm_bwd(**t, **kw)
    frozen = flce.flce_block_norm_bwd(**t, **kw, flags=flce.SKIP_DW)
    assert frozen[2:] == (None, None, None) and all(torch.equal(a, b) for a, b in zip(frozen[:2], full[:2]))
    params = flce.flce_block_norm_bwd(**t, **kw, flags=flce.SKIP_DX)
    assert params[0] is None and all(torch.equal(a, b) for a, b in zip(params[1:], full[1:]))
    # a shared gate per sequence whose gradient is not wanted
    c = make(40, 300, "f32", 13, gate="sequence", per=6, kind="silu")
    kw, t = _kw(c), {k: _dev(c, k) for k in ("h", "dn", "dh", "y")}
    full = flce.flce_block_norm_bwd(**t, **kw)
    frozen = flce.flce_block_norm_bwd(**t, **kw, flags=flce.SKIP_DW)
    assert torch.equal(full[0], frozen[0]) and torch.equal(full[1], frozen[1]) and frozen[2] is None
    # without a norm behind the sum its gradient is passed on
    c = make(12, 64, "f32", 14, pre=False)
    dh = _dev(c, "dh")
    dx, dy, *_ = flce.flce_block_norm_bwd(dh=dh, y=_dev(c, "y"), scale=0.75)
    assert dx is dh and torch.equal(dy, dh * 0.75)


def test_rows_do_not_see_each_other():
    """An infinite or NaN row leaves the other rows as they were, also those in its workgroup and wavefront."""
    import paper_2410_10989_amd as flce
    for H in (64, 700, 5000):
        c = make(40, H, "f32", 15, post=True, gate="token", kind="sigmoid")
        x, y = _dev(c, "x"), _dev(c, "y")
        clean = flce.flce_block_norm_fwd(x, y, **_kw(c))
        y[17, H // 2] = float("nan")
        x[3, 0] = float("inf")
        dirty = flce.flce_block_norm_fwd(x, y, **_kw(c))
        keep = torch.ones(40, dtype=torch.bool, device="cuda")
        keep[17] = keep[3] = False
        for a, b in zip(clean, dirty):
            assert torch.equal(a[keep], b[keep])
        assert torch.isnan(dirty[0][17]).all() and torch.isinf(dirty[0][3, 0])
        h, dn, dh, y = (_dev(c, k) for k in ("h", "dn", "dh", "y"))
        clean = flce.flce_block_norm_bwd(h, dn, dh, y, **_kw(c))
        dn[17, 1] = float("nan")
        dirty = flce.flce_block_norm_bwd(h, dn, dh, y, **_kw(c))
        keep[3] = True
        for a, b in zip(clean[:3], dirty[:3]):
            assert torch.equal(a[keep], b[keep])


@pytest.mark.parametrize("variant", [dict(), dict(post=True), dict(post=True, gate="channel", kind="silu"),
                                     dict(post=True, gate="sequence", per=5, kind="tanh"), dict(gate="sequence", per=7),
                                     dict(post=True, gate="token", kind="sigmoid"), dict(pre=False, post=True, gate="channel")],
                         ids=_name)
def test_eps_of_zero_where_rows_do_not_fill_a_workgroup(variant):
    """1 / rms of the rows that are not there is infinite; the sums over rows must not see it.  Row counts on both
    sides of where one workgroup takes all rows (48 of up to 128 elements, 12 of up to 1024)."""
    for i, (rows, H) in enumerate([(5, 9), (17, 64), (50, 100), (131, 128), (5, 300), (13, 512), (70, 520), (11, 1000), (3, 2000)]):
        for dtype in ("bf16", "f32"):
            print(f"case eps=0 rows={rows} H={H} {dtype} {variant}", flush=True)
            c = make(rows, H, dtype, 300 + i, eps=0.0, **variant)
            check_forward(c)
            check_backward(c)


def test_rows_of_zeros_and_large_eps():
    c = make(6, 130, "f32", 16, post=True, eps=0.5)
    for k in ("x", "y", "h"):
        c[k][2] = 0
    check_forward(c)
    check_backward(c)


def test_gates_that_saturate():
    for kind in ("sigmoid", "silu", "tanh"):
        c = make(4, 96, "f32", 17, gate="token", kind=kind)
        c["gate"][0], c["gate"][1], c["gate"][2, ::2], c["gate"][3] = -60.0, 60.0, 9.0, c["gate"][3] * 1e-4
        c["gate"] = c["gate"].astype(np.float32).astype(np.float64)
        check_forward(c)
        check_backward(c)


def test_gradients_against_central_differences():
    """The kernels' gradients against differences of the 64-bit forward (steps of 1e-5: errors of 1e-9 and less)."""
    import paper_2410_10989_amd as flce
    c = make(9, 40, "f32", 18, post=True, gate="sequence", per=4, kind="silu")
    f = oracle.forward(c["x"], c["y"], c["gate"], c["gamma_post"], c["gamma_pre"], **c["opt"])
    c["h"] = f["h"].astype(np.float32).astype(np.float64)
    got = dict(zip(("x", "y", "gate", "gamma_post", "gamma_pre"),
                   flce.flce_block_norm_bwd(_dev(c, "h"), _dev(c, "dn"), _dev(c, "dh"), _dev(c, "y"), **_kw(c))))

    def loss():
        f = oracle.forward(c["x"], c["y"], c["gate"], c["gamma_post"], c["gamma_pre"], **c["opt"])
        return (f["h"] * c["dh"]).sum() + (f["n"] * c["dn"]).sum()

    g = np.random.Generator(np.random.Philox(key=[18, 1]))
    for name, t in got.items():
        t = t.double().cpu().numpy()
        for _ in range(12):
            i = tuple(g.integers(0, n) for n in t.shape)
            at = c[name][i]
            c[name][i] = at + 1e-5
            up = loss()
            c[name][i] = at - 1e-5
            num = (up - loss()) / 2e-5
            c[name][i] = at
            # h rounded to fp32 and fp32 arithmetic: 2^-17 of magnitudes of at most 100 times the largest gradient
            assert abs(t[i] - num) <= 1e-3 * np.abs(t).max(), (name, i)


def test_another_stream_and_the_same_bits_every_time():
    import paper_2410_10989_amd as flce
    c = make(1030, 1024, "bf16", 19, post=True, gate="sequence", per=100, kind="tanh")
    t, kw = {k: _dev(c, k) for k in ("h", "dn", "dh", "y")}, _kw(c)
    want = flce.flce_block_norm_bwd(**t, **kw)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    ws = torch.empty(flce.flce_block_norm_workspace_bytes(1030, 1024, torch.bfloat16, 100), dtype=torch.uint8, device="cuda")
    for _ in range(3):
        got = flce.flce_block_norm_bwd(**t, **kw, workspace=ws, stream=side)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_two_captured_graphs_with_workspaces_of_their_own():
    import paper_2410_10989_amd as flce
    cases = [make(300, 520, "bf16", 20 + i, post=True, gate="channel", kind="silu") for i in range(2)]
    graphs = []
    for c in cases:
        t, kw = {k: _dev(c, k) for k in ("h", "dn", "dh", "y")}, _kw(c)
        x = _dev(c, "x")
        ws = torch.empty(flce.flce_block_norm_workspace_bytes(300, 520, torch.bfloat16), dtype=torch.uint8, device="cuda")
        h, n = torch.empty_like(t["h"]), torch.empty_like(t["h"])
        outs = dict(dx=torch.empty_like(t["h"]), dy=torch.empty_like(t["h"]), dgate=torch.empty_like(kw["gate"]),
                    dgamma_post=torch.empty_like(kw["gate"]), dgamma_pre=torch.empty_like(kw["gate"]))
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            flce.flce_block_norm_fwd(x, t["y"], **kw, h=h, n=n)
            flce.flce_block_norm_bwd(**t, **kw, **outs, workspace=ws)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            flce.flce_block_norm_fwd(x, t["y"], **kw, h=h, n=n)
            flce.flce_block_norm_bwd(**t, **kw, **outs, workspace=ws)
        graphs.append((graph, x, t, kw, [h, n, *outs.values()], ws))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for turn in range(4):
        for graph, x, t, kw, outs, _ in graphs:
            t["dn"].mul_(1.25)
            x.add_(0.5)
            for o in outs:
                o.fill_(float("nan"))
        torch.cuda.synchronize()
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g[0].replay()
        torch.cuda.synchronize()
        for graph, x, t, kw, outs, _ in graphs:
            want = [*flce.flce_block_norm_fwd(x, t["y"], **kw), *flce.flce_block_norm_bwd(**t, **kw)]
            assert all(torch.equal(a, b) for a, b in zip(outs, want)), turn


def test_a_graph_on_the_shared_workspace_outlives_its_growth():
    import paper_2410_10989_amd as flce
    flce.flce_release_workspace()
    c = make(600, 520, "bf16", 28, post=True, gate="channel", kind="silu")
    t, kw = {k: _dev(c, k) for k in ("h", "dn", "dh", "y")}, _kw(c)
    outs = dict(dx=torch.empty_like(t["h"]), dy=torch.empty_like(t["h"]), dgate=torch.empty_like(kw["gate"]),
                dgamma_post=torch.empty_like(kw["gate"]), dgamma_pre=torch.empty_like(kw["gate"]))
    flce.flce_block_norm_bwd(**t, **kw, **outs)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        flce.flce_block_norm_bwd(**t, **kw, **outs)
    big = make(2000, 4096, "bf16", 29, post=True)
    check_backward(big)   # needs more workspace
    for turn in range(3):
        t["dn"].mul_(1.25)
        for o in outs.values():
            o.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = flce.flce_block_norm_bwd(**t, **kw)
        assert all(torch.equal(a, b) for a, b in zip(outs.values(), want)), turn
    del graph
    flce.flce_release_workspace()


def test_rows_beyond_32_bit_offsets():
    """1200 rows, 2^21 elements apart: offsets of 5 GB and more than 2^31 elements."""
    import paper_2410_10989_amd as flce
    rows, H, ld = 1200, 72, 1 << 21
    c = make(rows, H, "bf16", 24, post=True, gate="token", kind="sigmoid")
    wide = torch.empty(rows * ld, dtype=torch.bfloat16, device="cuda").view(rows, ld)
    at = iter(range(0, ld, 128))

    def far(name):
        v = wide[:, (k := next(at)):k + H]
        v.copy_(torch.from_numpy(c[name]) if isinstance(name, str) else torch.full((rows, H), float("nan")))
        return v

    kw = _kw(c)
    kw["gate"] = far("gate")
    h, n = flce.flce_block_norm_fwd(far("x"), far("y"), **kw, h=far(None), n=far(None))
    ref = oracle.forward(c["x"], c["y"], c["gate"], c["gamma_post"], c["gamma_pre"], **c["opt"])
    _check("h", h, ref, "bf16")
    _check("n", n, ref, "bf16")
    got = flce.flce_block_norm_bwd(far("h"), far("dn"), far("dh"), far("y"), **kw, dx=far(None), dy=far(None), dgate=far(None))
    ref = reference_backward(c)
    for name, t in zip(("dx", "dy", "dgate", "dgamma_post", "dgamma_pre"), got):
        _check(name, t, ref, "bf16", rows_summed(c, name))


def test_a_very_long_row():
    """2^20 + 3 elements: sums of 1024 terms one after the other per thread, 2^-14 instead of 2^-19 (see above)."""
    import paper_2410_10989_amd as flce
    H, arith = (1 << 20) + 3, 2.0 ** -12
    c = make(2, H, "bf16", 26, post=True, gate="channel", kind="silu")
    ref = oracle.forward(c["x"], c["y"], c["gate"], c["gamma_post"], c["gamma_pre"], **c["opt"])
    h, n = flce.flce_block_norm_fwd(_dev(c, "x"), _dev(c, "y"), **_kw(c))
    _check("h", h, ref, "bf16", 0, arith)
    _check("n", n, ref, "bf16", 0, arith)
    ref = reference_backward(c)
    got = flce.flce_block_norm_bwd(_dev(c, "h"), _dev(c, "dn"), _dev(c, "dh"), _dev(c, "y"), **_kw(c))
    for name, t in zip(("dx", "dy", "dgate", "dgamma_post", "dgamma_pre"), got):
        _check(name, t, ref, "bf16", rows_summed(c, name), arith)


def test_binding_refusals():
    import paper_2410_10989_amd as flce
    x = torch.zeros(4, 8, device="cuda")
    g = torch.ones(8, device="cuda")
    bad = [dict(y=x.bfloat16()), dict(y=x[:3]), dict(y=x.cpu()), dict(y=x, gamma_pre=g[:7]), dict(y=x, gate=g, rows_per_gate=2),
           dict(y=x, gate=x), dict(y=x, gate_act="relu"), dict(y=x, rows_per_gate=-1), dict(y=x[:1].expand(4, 8)),
           dict(y=torch.zeros(8, 4, device="cuda").t())]
    for kw in bad:
        with pytest.raises((ValueError, TypeError)):
            flce.flce_block_norm_fwd(x, **kw)
    with pytest.raises(ValueError):
        flce.flce_block_norm_bwd(x, x.clone(), gamma_pre=g, flags=4)
    with pytest.raises(ValueError):
        flce.flce_block_norm_bwd(dh=x)
    with pytest.raises(flce.FlceError) as e:
        flce.flce_block_norm_fwd(x, x.clone(), g, n=x)
    assert e.value.status == 7


def test_a_gradient_of_what_there_is_not_is_refused():
    """The buffer would be left as it was, without a word."""
    import paper_2410_10989_amd as flce
    x, g = torch.ones(4, 8, device="cuda"), torch.ones(8, device="cuda")
    buf, row = torch.empty_like(x), torch.empty_like(g)
    for kw in (dict(dy=buf), dict(y=x, dgate=row), dict(y=x, dgamma_post=row)):
        with pytest.raises(ValueError):
            flce.flce_block_norm_bwd(x, x, x, gamma_pre=g, **kw)
    with pytest.raises(ValueError):
        flce.flce_block_norm_bwd(dh=x, y=x, dgamma_pre=row)
    # what a flag leaves out may be passed all the same, as for the other calls
    assert flce.flce_block_norm_bwd(x, x, x, gamma_pre=g, dgamma_pre=row, flags=flce.SKIP_DW)[4] is None
