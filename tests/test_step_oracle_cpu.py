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
