"""64-bit definitions of the operators at the other end of the model and behind its gradients: embedding lookup and
its table's gradient, layer norm with the residual sum in front of it, Newton-Schulz orthogonalisation.  Plain numpy,
one formula after the other.  Each result comes with `_mag`: the sum of the magnitudes of the terms it was added up
from, which rounding errors are relative to."""
from __future__ import annotations

import numpy as np


def _live(tokens, V, ignore_index, first_token):
    v = tokens.astype(object) - first_token          # (no overflow)
    return np.array([t != ignore_index and 0 <= r < V for t, r in zip(tokens, v)], dtype=bool), v


def embedding(table, tokens, scale=1.0, ignore_index=-100, first_token=0):
    live, v = _live(tokens, len(table), ignore_index, first_token)
    out = np.zeros((len(tokens), table.shape[1]))
    for i in np.flatnonzero(live):
        out[i] = scale * table[int(v[i])]
    return out


def embedding_grad(dout, tokens, V, scale=1.0, ignore_index=-100, first_token=0, base=None):
    live, v = _live(tokens, V, ignore_index, first_token)
    grad, mag = np.zeros((V, dout.shape[1])), np.zeros((V, dout.shape[1]))
    for i in np.flatnonzero(live):
        grad[int(v[i])] += scale * dout[i]
        mag[int(v[i])] += abs(scale) * np.abs(dout[i])
    if base is not None:
        grad, mag = grad + base, mag + np.abs(base)
    return grad, mag, live


def layer_norm(x, y=None, gamma=None, beta=None, eps=1e-5):
    h = x if y is None else x + y
    d = h - h.mean(1, keepdims=True)
    r = 1 / np.sqrt((d * d).mean(1, keepdims=True) + eps)
    g = 1.0 if gamma is None else gamma
    n = d * r * g + (0.0 if beta is None else beta)
    size = np.abs(x) if y is None else np.abs(x) + np.abs(y)
    n_mag = (size + size.mean(1, keepdims=True)) * r * np.abs(g) + np.abs(d * r * g) + (0.0 if beta is None else np.abs(beta))
    return dict(h=h, h_mag=size, n=n, n_mag=n_mag)


def layer_norm_grad(h, dn, dh=None, gamma=None, eps=1e-5):
    H = h.shape[1]
    d = h - h.mean(1, keepdims=True)
    r = 1 / np.sqrt((d * d).mean(1, keepdims=True) + eps)
    xh = d * r
    u = dn if gamma is None else dn * gamma
    mu, mx = u.mean(1, keepdims=True), (u * xh).mean(1, keepdims=True)
    base = 0.0 if dh is None else dh
    dx = base + r * (u - mu - xh * mx)
    # what an error of xh (of the size of h and its mean, times r) does, and the terms themselves
    xh_mag = np.abs(xh) + (np.abs(h) + np.abs(h).mean(1, keepdims=True)) * r
    ux = (np.abs(u) * xh_mag).mean(1, keepdims=True)
    dx_mag = np.abs(base) + r * (np.abs(u) + np.abs(u).mean(1, keepdims=True) + 2 * xh_mag * ux)
    return dict(dx=dx, dx_mag=dx_mag, dgamma=(dn * xh).sum(0), dgamma_mag=(np.abs(dn) * xh_mag).sum(0),
                dbeta=dn.sum(0), dbeta_mag=np.abs(dn).sum(0))


COEFFICIENTS = (3.4445, -4.7750, 2.0315)


def orthogonalize(G, steps=5, coefficients=COEFFICIENTS, scale=1.0, eps=1e-7):
    """coefficients: one triple for all steps, or one per step."""
    c = np.broadcast_to(np.asarray(coefficients, dtype=np.float64), (steps, 3))
    X = G / (np.sqrt((G * G).sum()) + eps)
    tall = X.shape[0] > X.shape[1]
    X = X.T if tall else X
    for a, b, q in c:
        A = X @ X.T
        X = a * X + (b * A + q * (A @ A)) @ X
    X = X.T if tall else X
    return scale * X


def orthogonalize_rounded(G, planes, steps=5, coefficients=COEFFICIENTS, scale=1.0, eps=1e-7):
    """The same with the roundings of a computation on fp16 operands, for the size of the error they make: X in two fp16
    planes, A and B in `planes`, products of the first planes (planes = 1) or hi hi + hi lo + lo hi (2), sums in
    fp32.  Scaled by 2^13, which keeps what is rounded in the type's normal range."""
    S = 2.0 ** 13
    c = np.broadcast_to(np.asarray(coefficients, dtype=np.float64), (steps, 3))

    def split(v):
        hi = (v.astype(np.float32) * np.float32(S)).astype(np.float16)
        lo = (v.astype(np.float32) * np.float32(S) - hi.astype(np.float32)).astype(np.float16)
        return hi.astype(np.float32) / np.float32(S), lo.astype(np.float32) / np.float32(S)

    def product(p, q):
        r = p[0] @ q[0]
        return r if planes == 1 else r + (p[0] @ q[1] + p[1] @ q[0])

    X = G / (np.sqrt((G * G).sum()) + eps)
    tall = X.shape[0] > X.shape[1]
    X = split(X.T if tall else X)
    for a, b, q in c.astype(np.float32):
        A = split(product(X, (X[0].T, X[1].T)))
        A = A if planes == 2 else (A[0], np.zeros_like(A[1]))
        B = split(b * (A[0] + A[1]) + q * product(A, A))
        X = a * (X[0] + X[1]) + product(B, X)
        last, X = X, split(X)
    last = last.T if tall else last
    return scale * last.astype(np.float64)
