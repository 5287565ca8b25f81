"""The 64-bit definition of the norms around a block against automatic differentiation and
central differences, and the host-side refusals of its entry points and of gradient clipping."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2410_10989_amd as flce
from oracle import block_norm_oracle as oracle


def _case(rows, H, seed, x=True, y=True, pre=True, post=False, gate="none", kind="linear"):
    g = np.random.Generator(np.random.Philox(key=[seed, 7]))
    per = {"none": 0, "channel": 0, "sequence": 3, "token": 1}[gate]
    shape = (H,) if per == 0 else (-(-rows // per), H)
    c = dict(x=g.standard_normal((rows, H)) if x else None, y=g.standard_normal((rows, H)) if y else None,
             gate=g.standard_normal(shape) if gate != "none" else None,
             gamma_post=1 + 0.2 * g.standard_normal(H) if post else None,
             gamma_pre=1 + 0.2 * g.standard_normal(H) if pre else None)
    opt = dict(kind=kind, rows_per_gate=per, scale=0.7, eps=1e-3)
    return c, opt, g.standard_normal((rows, H)), g.standard_normal((rows, H))


CASES = [dict(), dict(post=True), dict(gate="channel", kind="tanh"), dict(post=True, gate="sequence", kind="silu"),
         dict(post=True, gate="token", kind="sigmoid"), dict(x=False, post=True, gate="channel"),
         dict(pre=False, post=True, gate="sequence", kind="linear"), dict(y=False)]


def _loss(c, opt, dn, dh):
    """sum(h dh) + sum(n dn) of the forward."""
    f = oracle.forward(c["x"], c["y"], c["gate"], c["gamma_post"], c["gamma_pre"], **opt)
    h = f["h"] if c["y"] is not None else c["x"]
    return (h * dh).sum() + ((f["n"] * dn).sum() if c["gamma_pre"] is not None else 0.0)


def _backward(c, opt, dn, dh):
    f = oracle.forward(c["x"], c["y"], c["gate"], c["gamma_post"], c["gamma_pre"], **opt)
    h = f["h"] if c["y"] is not None else c["x"]
    pre = c["gamma_pre"] is not None
    b = oracle.backward(h if pre else None, dn if pre else None, dh, c["y"], c["gate"], c["gamma_post"], c["gamma_pre"], **opt)
    return {"x": b.get("dx"), "y": b.get("dy"), "gate": b.get("dgate"), "gamma_post": b.get("dgamma_post"),
            "gamma_pre": b.get("dgamma_pre")}


@pytest.mark.parametrize("kw", CASES)
def test_backward_is_the_derivative_of_the_forward(kw):
    c, opt, dn, dh = _case(7, 5, 11, **kw)
    grads = _backward(c, opt, dn, dh)
    step = 1e-5
    for name, v in c.items():
        if v is None:
            continue
        num = np.zeros_like(v)
        for i in np.ndindex(v.shape):
            at = v[i]
            v[i] = at + step
            up = _loss(c, opt, dn, dh)
            v[i] = at - step
            num[i] = (up - _loss(c, opt, dn, dh)) / (2 * step)
            v[i] = at
        # central differences: a third of step^2 times third derivatives, and roundings of 1e-16 * |loss| / step
        assert np.abs(num - grads[name]).max() <= 1e-7 * (1 + np.abs(num).max()), name


@pytest.mark.parametrize("kw", CASES)
def test_backward_agrees_with_automatic_differentiation(kw):
    c, opt, dn, dh = _case(13, 9, 12, **kw)
    grads = _backward(c, opt, dn, dh)
    t = {k: None if v is None else torch.from_numpy(v).requires_grad_() for k, v in c.items()}

    def norm(v, gamma):
        return torch.nn.functional.rms_norm(v, v.shape[1:], gamma, opt["eps"])

    h = t["x"]
    if t["y"] is not None:
        z = norm(t["y"], t["gamma_post"]) if t["gamma_post"] is not None else t["y"]
        if t["gate"] is not None:
            a = {"linear": lambda g: g, "sigmoid": torch.sigmoid, "silu": torch.nn.functional.silu, "tanh": torch.tanh}[opt["kind"]](t["gate"])
            z = z * (a if opt["rows_per_gate"] == 0 else a.repeat_interleave(opt["rows_per_gate"], 0)[:len(z)])
        h = opt["scale"] * z if h is None else h + opt["scale"] * z
    loss = (h * torch.from_numpy(dh)).sum()
    if t["gamma_pre"] is not None:
        loss = loss + (norm(h, t["gamma_pre"]) * torch.from_numpy(dn)).sum()
    loss.backward()
    for name, v in t.items():
        if v is not None:
            assert np.allclose(v.grad.numpy(), grads[name], rtol=1e-11, atol=1e-12), name


def test_activations_keep_their_accuracy_where_they_saturate():
    g = np.array([-40.0, -9.0, -1e-9, 0.0, 1e-9, 9.0, 40.0])
    for kind in oracle.ACTS:
        t = torch.from_numpy(g).requires_grad_()
        a = {"linear": lambda v: v, "sigmoid": torch.sigmoid, "silu": torch.nn.functional.silu, "tanh": torch.tanh}[kind](t)
        a.sum().backward()
        got = oracle.act(kind, g)
        assert np.allclose(got[0], a.detach().numpy(), rtol=1e-13, atol=0)
        assert np.allclose(got[1], t.grad.numpy(), rtol=1e-6, atol=1e-15)   # (torch's derivatives cancel)


# ---- refusals: found on the host, so host memory stands in for the device's ----

def _memory():
    buf = (ctypes.c_char * (1 << 16))()
    a = ctypes.addressof(buf)
    return buf, a + (-a) % 256


def _args(**kw):
    b = flce.FlceBlockNorm()
    b.size, b.rows, b.H, b.dtype, b.scale, b.eps = ctypes.sizeof(flce.FlceBlockNorm), 4, 8, 1, 1.0, 1e-6
    for k, v in kw.items():
        setattr(b, k, v)
    return b


BAD_ARGS = [(dict(size=8), 7), (dict(rows=0), 2), (dict(rows=2 ** 30 + 1), 2), (dict(H=0), 2), (dict(H=2 ** 24 + 1), 2),
            (dict(dtype=2), 3), (dict(gate_act=4), 7), (dict(gate_act=-1), 7), (dict(rows_per_gate=-1), 7),
            (dict(eps=-1.0), 7), (dict(eps=float("nan")), 7), (dict(scale=float("inf")), 7), (dict(ldx=7), 2),
            (dict(ldy=-8), 2), (dict(ldh=7), 2), (dict(ldn=1), 2), (dict(lddx=7), 2), (dict(lddn=2 ** 33), 2)]


@pytest.mark.parametrize("kw,status", BAD_ARGS)
def test_block_norm_refuses_bad_arguments(kw, status):
    buf, a = _memory()
    L = flce.lib()
    b = ctypes.byref(_args(**kw))
    assert L.flce_block_norm_fwd(a, a + 256, None, None, a + 512, b, a + 768, a + 1024, None) == status
    assert L.flce_block_norm_bwd(a, a + 256, a + 512, a + 768, None, None, a + 1024, b, a + 1280, a + 1536, None, None, a + 1792, None) == status
    assert L.flce_block_norm_workspace_bytes(b) == 0


def test_block_norm_refuses_missing_misaligned_and_overlapping_memory():
    buf, a = _memory()
    L = flce.lib()

    def fwd(x=a, y=a + 256, gate=None, post=None, pre=a + 512, h=a + 768, n=a + 1024, args=None, **kw):
        return L.flce_block_norm_fwd(x, y, gate, post, pre, ctypes.byref(args or _args(**kw)), h, n, None)

    assert L.flce_block_norm_fwd(a, a, None, None, None, None, a, a, None) == 1
    assert fwd(x=None, y=None) == 1 and fwd(h=None) == 1 and fwd(n=None) == 1
    assert fwd(y=None) == 7 and fwd(y=None, h=None, post=a) == 7 and fwd(y=None, h=None, gate=a) == 7
    assert fwd(pre=None) == 7 and fwd(y=None, h=None, pre=None, n=None) == 7
    assert fwd(x=a + 1) == 4 and fwd(n=a + 1025) == 4 and fwd(pre=a + 513) == 4
    assert fwd(h=a + 2) == 7 and fwd(h=a + 256) == 7 and fwd(n=a) == 7 and fwd(n=a + 768) == 7 and fwd(n=a + 512) == 7
    # columns of one wider buffer that lie beside each other do not overlap, columns that cut into each other do
    assert fwd(h=a + 256 + 14, ldy=16, ldh=16, rows=3) == 7
    assert fwd(h=a, ldx=16, ldh=17) == 7                         # x itself, but with another stride

    def bwd(h=a, dn=a + 256, dh=a + 512, y=a + 768, gate=None, post=None, pre=a + 1024, dx=a + 1280, dy=a + 1536,
            dgate=None, dpost=None, dpre=a + 1792, args=None, **kw):
        return L.flce_block_norm_bwd(h, dn, dh, y, gate, post, pre, ctypes.byref(args or _args(**kw)), dx, dy, dgate, dpost,
                                     dpre, None)

    assert bwd(h=None) == 1 and bwd(dn=None) == 1 and bwd(y=None) == 1
    assert bwd(y=None, dy=None, gate=a + 2048) == 1 and bwd(y=None, dy=None, post=a + 2048) == 1
    assert bwd(pre=None) == 7 and bwd(pre=None, h=None, dn=None, dh=None, dpre=None) == 1
    assert bwd(dgate=a + 2048) == 7 and bwd(dpost=a + 2048) == 7
    assert bwd(dx=None, dy=None, dpre=None) == 7
    assert bwd(dy=a + 1537) == 4 and bwd(dh=a + 513) == 4
    assert bwd(dx=a) == 7 and bwd(dx=a + 514) == 7 and bwd(dy=a + 512) == 7 and bwd(dy=a + 1280) == 7 and bwd(dpre=a + 1024) == 7
    assert bwd(workspace=a + 2050, workspace_bytes=1 << 20) == 4
    # rows that do not fit registers: 4 H bytes for each of the shared gradients at the least
    long = (ctypes.c_char * (4 << 20))()
    w = ctypes.addressof(long)
    w += (-w) % 256
    at = lambda k: w + (1 << 18) * k

    def rows_of_17000(nbytes, gate=None, post=None):
        b = _args(H=17000, workspace=at(13), workspace_bytes=nbytes)
        return L.flce_block_norm_bwd(at(0), at(1), at(2), at(3), gate, post, at(4), ctypes.byref(b), at(5), at(6),
                                     at(7) if gate else None, at(8) if post else None, at(9), None)

    for sets, gate, post in ((1, None, None), (2, at(10), None), (3, at(10), at(11))):
        assert rows_of_17000(4 * 17000 * sets - 1, gate, post) == 5


def test_h_on_x_excuses_no_other_input():
    """h may lie on x; a vector that is one of x's rows, or y with rows of another length from the same address, would
    be overwritten by h while other rows still need it."""
    buf, a = _memory()
    L = flce.lib()

    def fwd(x=a, y=a + 256, gate=None, post=None, pre=a + 512, h=a, n=a + 1024, **kw):
        return L.flce_block_norm_fwd(x, y, gate, post, pre, ctypes.byref(_args(**kw)), h, n, None)

    assert fwd(pre=a) == 7 and fwd(post=a) == 7
    assert fwd(gate=a) == 7 and fwd(gate=a, rows_per_gate=2) == 7 and fwd(gate=a, rows_per_gate=1, ldgate=16) == 7
    assert fwd(y=a, ldy=16) == 7 and fwd(y=a, ldx=16, ldh=16) == 7
    assert fwd(rows=1, pre=a) == 7 and fwd(rows=1, post=a) == 7


def test_block_norm_backward_refuses_a_workspace_on_its_operands():
    L = flce.lib()
    big = (ctypes.c_char * (2 << 20))()
    w = ctypes.addressof(big)
    w += (-w) % 256
    rows, H = 64, 64   # 8 KB per bf16 matrix; more rows than one workgroup takes without partial sums
    at = [w + 8192 * k for k in range(9)]
    need = flce.flce_block_norm_workspace_bytes(rows, H, torch.bfloat16)
    assert 256 < need <= 1 << 20

    def bwd(ws, nbytes=need, **kw):
        b = _args(rows=rows, H=H, workspace=ws, workspace_bytes=nbytes, **kw)
        return L.flce_block_norm_bwd(at[0], at[1], at[2], at[3], at[4], at[5], at[5] + 256, ctypes.byref(b), at[6], at[7],
                                     at[8], at[8] + 256, at[8] + 512, None)

    for operand in (*at[:6], at[5] + 256, *at[6:], at[8] + 256, at[8] + 512):
        assert bwd(operand) == 7 and bwd(operand - 256 if operand > w else operand) == 7


def test_vectors_between_the_rows_of_a_matrix_do_not_overlap_it():
    """A single row against rows that lie apart: only shared bytes count.  (Refusals behind the overlap check show
    that a call passed it: a workspace off its alignment.)"""
    L = flce.lib()
    big = (ctypes.c_char * (1 << 16))()
    w = ctypes.addressof(big)
    w += (-w) % 256

    def bwd(dpre, ldh=64, **kw):   # h: 4 rows of 16 bytes, 128 bytes apart
        b = _args(rows=4, ldh=ldh, workspace=w + 8194, workspace_bytes=1 << 12, **kw)
        return L.flce_block_norm_bwd(w + 256, w + 1024, w + 2048, w + 3328, None, None, w + 4096, ctypes.byref(b), w + 5120,
                                     w + 6144, None, None, dpre, None)

    first = w + 256
    for dpre in (first + 16, first + 112, first + 128 + 16, first + 2 * 128 + 112, first + 3 * 128 + 16, first - 16):
        assert bwd(dpre) == 4
    for dpre in (first - 2, first, first + 14, first + 114, first + 128, first + 128 + 14, first + 3 * 128 + 14, first + 2 * 128 + 114):
        assert bwd(dpre) == 7
    assert bwd(first + 3 * 128 - 12, ldh=64) == 7 and bwd(first + 4, ldh=64) == 7


def test_block_norm_workspace_is_bounded():
    need = [flce.flce_block_norm_workspace_bytes(rows, 4096, torch.bfloat16, per)
            for rows in (1, 1000, 10 ** 6, 2 ** 30) for per in (0, 1, 5, 2048)]
    assert all(n <= 128 << 20 for n in need) and all(n >= 8 * 4096 for n in need[4:])
    assert flce.flce_block_norm_workspace_bytes(2 ** 30, 2 ** 24, torch.float32) <= 3 * 256 * 2 ** 24 * 4
    assert flce.flce_block_norm_workspace_bytes(0, 8, torch.float32) == 0


def test_clipping_refuses_bad_arguments():
    buf, a = _memory()
    L = flce.lib()
    V2, C2, D2 = ctypes.c_void_p * 2, ctypes.c_int64 * 2, ctypes.c_int * 2
    grads, outs = V2(a, a + 256), V2(a + 512, a + 768)

    def clip(g=grads, o=outs, c=C2(8, 8), d=D2(0, 1), n=2, kind=0, most=1.0, norm=a + 1024, ws=a + 2048, size=1 << 15):
        return L.flce_clip_grad_norm(g, o, c, d, n, kind, ctypes.c_float(most), norm, ws, size, None)

    assert clip(g=None) == 1 and clip(c=None) == 1 and clip(d=None) == 1 and clip(norm=None) == 1
    assert clip(g=V2(a, None)) == 1 and clip(o=V2(a + 512, None)) == 1
    assert clip(n=-1) == 7 and clip(kind=2) == 7 and clip(most=-1.0) == 7 and clip(most=float("nan")) == 7
    assert clip(most=float("inf")) == 7
    assert clip(c=C2(8, -1)) == 2 and clip(c=C2(2 ** 41, 8)) == 2 and clip(d=D2(0, 2)) == 3
    assert clip(g=V2(a + 2, a + 256)) == 4 and clip(g=V2(a, a + 257)) == 4 and clip(norm=a + 1026) == 4
    assert clip(ws=a + 2050) == 4 and clip(size=8) == 5
    assert flce.lib().flce_grad_norm_workspace_bytes(2) <= 1 << 15
    assert clip(g=V2(a, a), o=None) == 7                             # the same gradient twice, in place
    assert clip(g=V2(a, a + 16), o=None, d=D2(0, 0)) == 7            # ... or half of it
    assert clip(o=V2(a + 512, a + 512)) == 7                         # two outputs in one place
    assert clip(o=V2(a + 16, a + 768)) == 7                          # an output on half of its own input
    assert clip(o=V2(a + 512, a)) == 7                               # ... or on another's
    L1 = (ctypes.c_float * 1)(0.5)
    assert L.flce_grad_clip(grads, outs, C2(8, 8), D2(0, 1), 2, None, ctypes.c_float(1.0), None) == 1
    assert L.flce_grad_clip(V2(a, a), None, C2(8, 8), D2(0, 0), 2, a + 1024, ctypes.c_float(1.0), None) == 7
    assert L.flce_grad_norm(grads, C2(8, 8), D2(0, 1), 2, 5, a + 1024, a + 2048, 1 << 15, None) == 7
    assert L.flce_grad_norm(grads, C2(8, 8), D2(0, 1), 2, 0, None, a + 2048, 1 << 15, None) == 1
    assert L.flce_grad_norm(grads, C2(8, 8), D2(0, 1), 2, 0, a + 1024, a + 2048, 8, None) == 5
    del L1


def test_clipping_refuses_a_norm_or_workspace_inside_a_tensor():
    """The norm is written (or read) by one workgroup while others scale the tensors and read the partial results."""
    buf, a = _memory()
    L = flce.lib()
    V2, C2, D2 = ctypes.c_void_p * 2, ctypes.c_int64 * 2, ctypes.c_int * 2
    # tensors of 16000 and 4000 bytes
    grads, outs, counts, dtypes = V2(a, a + 16384), V2(a + 20480, a + 36864), C2(4000, 2000), D2(0, 1)
    ws, size = a + 45056, 16384
    most = ctypes.c_float(1.0)

    def clip(norm, o=outs, ws=ws):
        return L.flce_clip_grad_norm(grads, o, counts, dtypes, 2, 0, most, norm, ws, size, None)

    for inside in (a, a + 15996, a + 16384, a + 20380, a + 20480, a + 36864 + 3996):
        assert clip(inside) == 7
    for inside in (a, a + 15996, a + 16384):
        assert clip(inside, o=None) == 7
        assert L.flce_grad_clip(grads, None, counts, dtypes, 2, inside, most, None) == 7
        assert L.flce_grad_norm(grads, counts, dtypes, 2, 0, inside, ws, size, None) == 7
    assert L.flce_grad_clip(grads, outs, counts, dtypes, 2, a + 20480, most, None) == 7
    big = (ctypes.c_char * (1 << 20))()
    w = ctypes.addressof(big)
    w += (-w) % 256
    counts = C2(100_000, 2000)
    grads, outs = V2(w, w + 401408), V2(w + 409600, w + 811008)
    for inside in (w, w + 399872, w + 401408, w + 809472):
        assert clip(a, ws=inside) == 7
    assert clip(a + 4096, ws=a) == 7 and L.flce_grad_norm(grads, counts, dtypes, 2, 0, a, a, size, None) == 7
    assert L.flce_grad_norm(grads, counts, dtypes, 2, 1, a, w + 256, size, None) == 7


def test_binding_refuses_what_the_library_cannot_see():
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError):
        flce.flce_block_norm_fwd(x, x, torch.ones(8))
    with pytest.raises(ValueError):
        flce.flce_block_norm_fwd(None, None)
    with pytest.raises(ValueError):
        flce.flce_block_norm_bwd(dn=x, h=x, gamma_pre=torch.ones(8))
    with pytest.raises(ValueError):
        flce.flce_grad_norm([x])
    with pytest.raises(ValueError):
        flce.flce_clip_grad_norm([], 1.0)


def test_clipping_by_a_norm_needs_one():
    """None would be memory that nobody has written."""
    for grads in ([torch.zeros(3)], []):
        with pytest.raises(ValueError, match="norm must be one float32 value"):
            flce.flce_grad_clip(grads, None, 1.0)


def test_clip_definition():
    t = [np.array([3.0, -4.0]), np.array([[12.0]])]
    assert oracle.grad_norm(t) == 13.0 and oracle.grad_norm(t, "inf") == 12.0
    assert oracle.clip_factor(13.0, 26.0) == 1.0 and abs(oracle.clip_factor(13.0, 6.5) - 0.5) < 1e-7
    assert oracle.clip_factor(np.inf, 1.0) == 1.0 and oracle.clip_factor(np.nan, 1.0) == 1.0
    ref = [torch.nn.Parameter(torch.zeros(2, dtype=torch.float64)), torch.nn.Parameter(torch.zeros(1, 1, dtype=torch.float64))]
    for p, g in zip(ref, t):
        p.grad = torch.from_numpy(g.copy())
    norm = torch.nn.utils.clip_grad_norm_(ref, 5.0)
    f = oracle.clip_factor(oracle.grad_norm(t), 5.0)
    assert abs(float(norm) - 13.0) < 1e-12 and all(np.allclose(p.grad.numpy(), g * f, rtol=1e-14) for p, g in zip(ref, t))
