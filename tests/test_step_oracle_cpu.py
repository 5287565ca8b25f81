"""The 64-bit definitions of the embedding, the layer norm and the orthogonalisation against automatic
differentiation, differences and the singular value decomposition, and the host-side refusals of their entry points."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2410_10989_amd as flce
from oracle import step_oracle as oracle


def rng(*key):
    return np.random.Generator(np.random.Philox(key=list(key)))


def test_embedding_gradient_is_the_derivative_of_the_lookup():
    g = rng(1, 2)
    table, tokens = g.standard_normal((11, 5)), g.integers(0, 14, 40)
    tokens[3] = -100
    dout = g.standard_normal((40, 5))
    grad, mag, live = oracle.embedding_grad(dout, tokens, 11, 1.7, -100, 2)
    t = torch.from_numpy(table).requires_grad_()
    at = torch.from_numpy(tokens - 2)
    ok = (at >= 0) & (at < 11)
    out = torch.where(ok[:, None], 1.7 * t[at.clamp(0, 10)], torch.zeros(()).double())
    assert np.array_equal(live, ok.numpy())
    np.testing.assert_allclose(oracle.embedding(table, tokens, 1.7, -100, 2), out.detach().numpy(), rtol=1e-15)
    out.backward(torch.from_numpy(dout))
    np.testing.assert_allclose(grad, t.grad.numpy(), rtol=1e-13, atol=1e-14)
    base = g.standard_normal((11, 5))
    np.testing.assert_allclose(oracle.embedding_grad(dout, tokens, 11, 1.7, -100, 2, base)[0], grad + base)
    assert (mag >= np.abs(grad) - 1e-12).all()


def test_embedding_with_an_ignored_token_inside_the_table():
    table = np.arange(12.0).reshape(4, 3)
    assert (oracle.embedding(table, np.array([1, 2, 1]), 1.0, 2)[1] == 0).all()


# ---- refusals, before anything touches a device ----

def embedding_args(**kw):
    d = dict(size=ctypes.sizeof(flce.FlceEmbedding), rows=6, V=9, H=8, dtype=flce.FLCE_F32, accumulate=0, first_token=0,
             ignore_index=-100, scale=1.0)
    d.update(kw)
    return flce.FlceEmbedding(**d)


A = 1 << 20   # addresses that are only compared
E = dict(table=A, tokens=2 * A, out=3 * A)
EMBEDDING_REFUSED = [
    (dict(size=8), {}, 7), (dict(rows=0), {}, 2), (dict(rows=(1 << 30) + 1), {}, 2), (dict(V=0), {}, 2), (dict(V=(1 << 30) + 1), {}, 2),
    (dict(H=0), {}, 2), (dict(H=(1 << 24) + 1), {}, 2), (dict(dtype=2), {}, 3), (dict(scale=float("inf")), {}, 7),
    (dict(scale=float("nan")), {}, 7), (dict(ldtable=7), {}, 2), (dict(ldrows=-8), {}, 2), (dict(ldrows=7), {}, 2),
    ({}, dict(table=0), 1), ({}, dict(tokens=0), 1), ({}, dict(out=0), 1), ({}, dict(table=A + 2), 4), ({}, dict(tokens=2 * A + 4), 4),
    ({}, dict(out=3 * A + 1), 4), ({}, dict(out=A), 7), ({}, dict(out=A + 9 * 32 - 4), 7)]


@pytest.mark.parametrize("kw,ptr,status", EMBEDDING_REFUSED)
def test_embedding_refusals(kw, ptr, status):
    p = dict(E, **ptr)
    a = embedding_args(**kw)
    L = flce.lib()
    assert L.flce_embedding_fwd(p["table"], p["tokens"], ctypes.byref(a), p["out"], None) == status
    # the backward: dout [rows, H] in place of out, dtable [V, H] in place of the table
    assert L.flce_embedding_bwd(p["out"], p["tokens"], ctypes.byref(a), p["table"], None) == status


def test_embedding_backward_refusals():
    L = flce.lib()
    for out in (2 * A + 40, 2 * A - 6 * 32 + 4):   # the lookup's output on the tokens
        assert L.flce_embedding_fwd(A, 2 * A, ctypes.byref(embedding_args()), out, None) == 7
    call = lambda a, dout=A, tokens=2 * A, dtable=3 * A: L.flce_embedding_bwd(dout, tokens, ctypes.byref(a) if a else None, dtable, None)
    assert call(None) == 1
    assert call(embedding_args(accumulate=2)) == 7
    need = flce.flce_embedding_workspace_bytes(6, 9, 8, torch.float32)
    assert need > 0
    assert call(embedding_args(workspace=4 * A + 8, workspace_bytes=need)) == 4
    assert call(embedding_args(workspace=4 * A, workspace_bytes=need - 1)) == 5
    for at in (A, 2 * A, 3 * A):   # on dout, the tokens, the gradient
        assert call(embedding_args(workspace=at, workspace_bytes=need)) == 7
    assert call(embedding_args(), tokens=3 * A + 8) == 7
    assert flce.flce_embedding_workspace_bytes(0, 9, 8, torch.float32) == 0


def test_embedding_binding_refusals():
    t = torch.zeros(4, 8)
    with pytest.raises(ValueError):
        flce.flce_embedding_fwd(t, torch.zeros(3, dtype=torch.int64))      # not on the GPU
    with pytest.raises(TypeError):
        flce.flce_embedding_fwd(t.half(), torch.zeros(3, dtype=torch.int64))
    with pytest.raises(ValueError):
        flce.flce_embedding_bwd(t, torch.zeros(4, dtype=torch.int64), 9)


# ---- layer norm ----

@pytest.mark.parametrize("y,gamma,beta,dh", [(True, True, True, True), (False, True, False, True), (True, False, True, False),
                                             (False, False, False, False)])
def test_layer_norm_gradient_is_the_derivative_of_the_forward(y, gamma, beta, dh):
    g = rng(3, 4)
    x, dn = g.standard_normal((4, 7)) + 2, g.standard_normal((4, 7))
    y = g.standard_normal((4, 7)) if y else None
    gamma, beta = g.standard_normal(7) if gamma else None, g.standard_normal(7) if beta else None
    dh = g.standard_normal((4, 7)) if dh else None
    f = oracle.layer_norm(x, y, gamma, beta, 1e-3)
    leaf = lambda a: None if a is None else torch.from_numpy(a).requires_grad_()
    X, G, B = leaf(x), leaf(gamma), leaf(beta)
    h = X if y is None else X + torch.from_numpy(y)
    n = torch.nn.functional.layer_norm(h, (7,), G, B, 1e-3)
    np.testing.assert_allclose(f["n"], n.detach().numpy(), rtol=1e-12, atol=1e-13)
    np.testing.assert_allclose(f["h"], h.detach().numpy())
    loss = (n * torch.from_numpy(dn)).sum() + (0 if dh is None else (h * torch.from_numpy(dh)).sum())
    loss.backward()
    b = oracle.layer_norm_grad(f["h"], dn, dh, gamma, 1e-3)
    np.testing.assert_allclose(b["dx"], X.grad.numpy(), rtol=1e-10, atol=1e-12)
    if gamma is not None:
        np.testing.assert_allclose(b["dgamma"], G.grad.numpy(), rtol=1e-11, atol=1e-12)
    if beta is not None:
        np.testing.assert_allclose(b["dbeta"], B.grad.numpy(), rtol=1e-11, atol=1e-12)
    assert all((b[k + "_mag"] >= np.abs(b[k]) - 1e-12).all() for k in ("dx", "dgamma", "dbeta"))


def layer_norm_args(**kw):
    d = dict(size=ctypes.sizeof(flce.FlceLayerNorm), rows=6, H=8, dtype=flce.FLCE_F32, eps=1e-5)
    d.update(kw)
    return flce.FlceLayerNorm(**d)


@pytest.mark.parametrize("kw,status", [
    (dict(size=8), 7), (dict(rows=0), 2), (dict(rows=(1 << 30) + 1), 2), (dict(H=0), 2), (dict(H=(1 << 24) + 1), 2), (dict(dtype=5), 3),
    (dict(eps=-1.0), 7), (dict(eps=float("nan")), 7), (dict(eps=float("inf")), 7), (dict(ldx=7), 2), (dict(ldn=-8), 2), (dict(lddx=3), 2)])
def test_layer_norm_refuses_bad_arguments(kw, status):
    a, L = layer_norm_args(**kw), flce.lib()
    assert L.flce_layer_norm_fwd(A, None, None, None, ctypes.byref(a), None, 2 * A, None) == status
    assert L.flce_layer_norm_bwd(A, 2 * A, None, None, ctypes.byref(a), 3 * A, None, None, None) == status
    assert flce.lib().flce_layer_norm_workspace_bytes(ctypes.byref(a)) == 0


def test_layer_norm_refuses_bad_pointers():
    L, a = flce.lib(), ctypes.byref(layer_norm_args())
    row = 6 * 8 * 4

    def fwd(x=A, y=2 * A, gamma=3 * A, beta=4 * A, h=5 * A, n=6 * A, args=a):
        return L.flce_layer_norm_fwd(x, y, gamma, beta, args, h, n, None)

    assert fwd(args=None) == 1 and fwd(x=None) == 1 and fwd(n=None) == 1 and fwd(h=None) == 1
    assert fwd(y=None) == 7                                       # h without y
    for k in ("x", "y", "gamma", "beta", "h", "n"):
        assert fwd(**{k: 7 * A + 2}) == 4
    assert fwd(h=6 * A) == 7 and fwd(h=6 * A + row - 4) == 7      # h and n
    assert fwd(n=A) == 7 and fwd(n=2 * A) == 7 and fwd(n=3 * A - row + 4) == 7 and fwd(n=4 * A) == 7
    assert fwd(h=A + 4) == 7 and fwd(h=2 * A) == 7 and fwd(h=3 * A) == 7

    def bwd(h=A, dn=2 * A, dh=3 * A, gamma=4 * A, dx=5 * A, dgamma=6 * A, dbeta=7 * A, args=a):
        return L.flce_layer_norm_bwd(h, dn, dh, gamma, args, dx, dgamma, dbeta, None)

    assert bwd(args=None) == 1 and bwd(h=None) == 1 and bwd(dn=None) == 1
    assert bwd(gamma=None) == 7 and bwd(dx=None, dgamma=None, dbeta=None) == 7
    for k in ("h", "dn", "dh", "gamma", "dx", "dgamma", "dbeta"):
        assert bwd(**{k: 8 * A + 1}) == 4
    for at in (A, 2 * A, 4 * A, 6 * A, 7 * A, 3 * A + 4, 3 * A - 4):
        assert bwd(dx=at) == 7
    for at in (A, 2 * A, 3 * A, 4 * A, 7 * A):
        assert bwd(dgamma=at) == 7
    # a workspace that lies on an operand, is too small, misaligned
    big = dict(rows=4000, H=8)
    need = flce.flce_layer_norm_workspace_bytes(4000, 8, torch.float32)
    assert need > 0
    for at in (A, 2 * A, 3 * A, 4 * A, 5 * A, 6 * A, 7 * A):
        assert bwd(args=ctypes.byref(layer_norm_args(workspace=at, workspace_bytes=need, **big))) == 7
    assert bwd(args=ctypes.byref(layer_norm_args(workspace=9 * A + 4, workspace_bytes=need, **big))) == 4
    long = dict(rows=6, H=20000)
    assert bwd(args=ctypes.byref(layer_norm_args(workspace=9 * A, workspace_bytes=8 * 20000 - 4, **long))) == 5


def test_layer_norm_binding_refusals():
    t = torch.zeros(4, 8)
    with pytest.raises(ValueError):
        flce.flce_layer_norm_fwd(t)
    with pytest.raises(ValueError):
        flce.flce_layer_norm_bwd(t, t)


# ---- orthogonalisation ----

@pytest.mark.parametrize("rows,cols", [(6, 9), (9, 6), (1, 4), (5, 5)])
def test_orthogonalisation_acts_on_the_singular_values(rows, cols):
    g = rng(5, rows)
    G = g.standard_normal((rows, cols))
    got = oracle.orthogonalize(G, scale=1.5)
    U, s, Vt = np.linalg.svd(G, full_matrices=False)
    s = s / (np.linalg.norm(G) + 1e-7)
    for _ in range(5):
        s = 3.4445 * s - 4.7750 * s ** 3 + 2.0315 * s ** 5
    np.testing.assert_allclose(got, 1.5 * (U * s) @ Vt, rtol=1e-9, atol=1e-10)
    # the cubic that converges: U V^T itself
    np.testing.assert_allclose(oracle.orthogonalize(G, 60, (1.5, -0.5, 0.0)), U @ Vt, atol=1e-9)


def test_rounded_orthogonalisation_is_near_the_exact_one():
    G = rng(6, 7).standard_normal((60, 90))
    ref = oracle.orthogonalize(G)
    err = [np.linalg.norm(oracle.orthogonalize_rounded(G, p) - ref) / np.linalg.norm(ref) for p in (1, 2)]
    assert 1e-5 < err[0] < 5e-3 and err[1] < 5e-6


def ortho_args(**kw):
    d = dict(size=ctypes.sizeof(flce.FlceOrthogonalizeArgs), rows=70, cols=90, dtype=flce.FLCE_F32, steps=5, coefficients=None, per_step=0,
             scale=1.0, eps=1e-7)
    d.update(kw)
    c = d.pop("coefficients")
    a = flce.FlceOrthogonalizeArgs(**d)
    if c is not None:
        a._keep = (ctypes.c_float * len(c))(*c)
        a.coefficients = ctypes.addressof(a._keep)
    return a


def ortho(a, ins=(A, 2 * A), outs=(3 * A, 4 * A), n=None):
    P = ctypes.c_void_p * 2
    return flce.lib().flce_orthogonalize(P(*ins) if ins else None, P(*outs) if outs else None, len(ins) if n is None else n,
                                         ctypes.byref(a) if a else None, None)


INF = float("inf")


@pytest.mark.parametrize("kw,status", [
    (dict(size=4), 7), (dict(rows=0), 2), (dict(cols=0), 2), (dict(rows=(1 << 20) + 1), 2), (dict(cols=(1 << 20) + 1), 2),
    (dict(rows=1 << 15, cols=(1 << 13) + 1), 2), (dict(dtype=7), 3), (dict(steps=0), 7), (dict(steps=33), 7), (dict(per_step=2), 7),
    (dict(scale=INF), 7), (dict(eps=-1e-9), 7), (dict(eps=float("nan")), 7), (dict(coefficients=[1.0, INF, 0.0]), 7),
    (dict(coefficients=[12.0, 0.0, 0.0]), 7),                                       # 12^3 > 1024
    (dict(coefficients=[3.0, 2.0, 1.0]), 7), (dict(steps=1, coefficients=[0.0, 0.0, 1025.0]), 7)])
def test_orthogonalisation_refuses_bad_arguments(kw, status):
    a = ortho_args(**kw)
    assert ortho(a) == status
    assert flce.lib().flce_orthogonalize_workspace_bytes(2, ctypes.byref(a)) == 0


def test_orthogonalisation_refuses_bad_pointers():
    size = 70 * 90 * 4
    need = flce.flce_orthogonalize_workspace_bytes(2, 70, 90, torch.float32)
    assert need > 0
    with_ws = lambda at=9 * A, n=need: ortho_args(workspace=at, workspace_bytes=n)
    assert ortho(None) == 1 and ortho(ortho_args(), ins=None, n=2) == 1
    assert ortho(ortho_args(), n=-1) == 7 and ortho(ortho_args(), n=0) == 0
    assert ortho(with_ws(), ins=(A, 0)) == 1 and ortho(with_ws(), outs=(0, A)) == 1
    assert ortho(with_ws(), ins=(A, 2 * A + 2)) == 4 and ortho(with_ws(), outs=(3 * A + 1, 4 * A)) == 4
    assert ortho(with_ws(at=9 * A + 64)) == 4
    assert ortho(with_ws(n=flce.flce_orthogonalize_workspace_bytes(1, 70, 90, torch.float32) - 1)) == 5
    assert ortho(with_ws(), outs=(3 * A, 3 * A)) == 7                       # two outs
    assert ortho(with_ws(), outs=(3 * A, 3 * A + size - 4)) == 7
    assert ortho(with_ws(), outs=(2 * A, A)) == 7                           # an out on another's in
    assert ortho(with_ws(), outs=(A + 4, 4 * A)) == 7                       # shifted on its own
    assert ortho(with_ws(), ins=(A, A), outs=None) == 7                     # the same matrix twice, in place
    for at in (A, 2 * A, 3 * A, 4 * A):
        assert ortho(with_ws(at=at)) == 7                                   # the workspace on a matrix


def test_orthogonalisation_accepts_what_stays_in_range():
    big = lambda **kw: flce.lib().flce_orthogonalize_workspace_bytes(1, ctypes.byref(ortho_args(**kw))) > 0
    assert big() and big(steps=32) and big(coefficients=[2.0, -1.5, 0.5], steps=32) and big(coefficients=[0.0, 0.0, 0.0])
    assert big(steps=1, coefficients=[1000.0, 0.0, 0.0]) and big(rows=1 << 15, cols=1 << 13) and big(rows=1 << 20, cols=1)
    assert big(steps=2, per_step=1, coefficients=[8.0, -22.0, 16.0, 4.0, -3.0, 0.5])


def test_orthogonalisation_binding_refusals():
    t = torch.zeros(4, 8)
    with pytest.raises(ValueError):
        flce.flce_orthogonalize([t])
    with pytest.raises(ValueError):
        flce.flce_orthogonalize([t, torch.zeros(8, 4)])
    assert flce.flce_orthogonalize([]) == []


def test_orthogonalisation_coefficients():
    from paper_2410_10989_amd.binding import _orthogonalize_args
    import numpy as np
    one, two = (2.0, -1.5, 0.5), [(8.0, -22.0, 16.0), (4.0, -3.0, 0.5)]
    for given in (one, list(one), np.array(one), torch.tensor(one)):
        args = _orthogonalize_args(4, 8, flce.FLCE_F32, 2, given, 1.0, 1e-7)
        assert args.per_step == 0 and list(args._coefficients) == list(one)
    for given in (two, np.array(two), torch.tensor(two)):
        args = _orthogonalize_args(4, 8, flce.FLCE_F32, 2, given, 1.0, 1e-7)
        assert args.per_step == 1 and list(args._coefficients) == [x for t in two for x in t]
    for given in ([], (1.0, 2.0), [(1.0, 2.0, 3.0)], two + two, torch.zeros(2, 2)):
        with pytest.raises(ValueError):
            _orthogonalize_args(4, 8, flce.FLCE_F32, 2, given, 1.0, 1e-7)
