"""64-bit numpy definition of the norms around a block and of gradient clipping (test infrastructure).

Beside every value stands the magnitude of what was added up to it (the same expression with every
term's absolute value): rounding errors of the kernels are bounded by multiples of that, not of the
value, where terms cancel.
"""
from __future__ import annotations

import numpy as np

ACTS = ("linear", "sigmoid", "silu", "tanh")


def act(kind: str, g):
    """a(g), a'(g)."""
    if kind == "linear":
        return g, np.ones_like(g)
    if kind == "tanh":
        a = np.tanh(g)
        return a, 1.0 / np.cosh(np.clip(g, -300, 300)) ** 2
    e = np.exp(-np.abs(g))
    sig, rest = np.where(g >= 0, 1, e) / (1 + e), np.where(g >= 0, e, 1) / (1 + e)
    if kind == "sigmoid":
        return sig, sig * rest
    return g * sig, sig * (1 + g * rest)


def gate_rows(gate, rows, rows_per_gate):
    """The gate row of every row."""
    return np.broadcast_to(gate, (rows, gate.shape[-1])) if rows_per_gate == 0 else gate[np.arange(rows) // rows_per_gate]


def rstd(v, eps):
    return 1.0 / np.sqrt((v * v).mean(1, keepdims=True) + eps)


def forward(x, y, gate=None, gamma_post=None, gamma_pre=None, kind="linear", rows_per_gate=0, scale=1.0, eps=1e-6):
    """{h, n} and their magnitudes {h_mag, n_mag}."""
    out = {}
    if y is not None:
        z = y if gamma_post is None else y * rstd(y, eps) * gamma_post
        if gate is not None:
            z = z * act(kind, gate_rows(gate, len(y), rows_per_gate))[0]
        z = scale * z
        h = z if x is None else x + z
        out["h"], mag = h, np.abs(z) + (0 if x is None else np.abs(x))
        out["h_mag"] = mag
    else:
        h, mag = x, np.abs(x)
    if gamma_pre is not None:
        r = rstd(h, eps)
        out["n"] = h * r * gamma_pre
        # an error of h moves n itself and the row's mean square
        length = np.sqrt((h * h).sum(1, keepdims=True)) + 1e-300
        out["n_mag"] = mag * r * np.abs(gamma_pre) + np.abs(out["n"]) * (1 + np.sqrt((mag * mag).sum(1, keepdims=True)) / length)
    return out


def backward(h, dn, dh, y, gate=None, gamma_post=None, gamma_pre=None, kind="linear", rows_per_gate=0, scale=1.0,
             eps=1e-6):
    """{dx, dy, dgate, dgamma_post, dgamma_pre} and their magnitudes (*_mag)."""
    out = {}
    like = dn if dn is not None else dh
    rows, H = like.shape
    D = np.zeros((rows, H)) if dh is None else dh.copy()
    mD = np.abs(D)
    if gamma_pre is not None:
        r = rstd(h, eps)
        xh, u = h * r, dn * gamma_pre
        D += r * (u - xh * (u * xh).mean(1, keepdims=True))
        mD += r * (np.abs(u) + np.abs(xh) * np.abs(u * xh).mean(1, keepdims=True))
        out["dgamma_pre"], out["dgamma_pre_mag"] = (dn * xh).sum(0), np.abs(dn * xh).sum(0)
    out["dx"], out["dx_mag"] = D, mD
    if y is None:
        return out
    q = rstd(y, eps) if gamma_post is not None else None
    z = y if gamma_post is None else y * q * gamma_post
    dz, mz = scale * D, abs(scale) * mD
    if gate is not None:
        a, da = act(kind, gate_rows(gate, rows, rows_per_gate))
        dg, mg = dz * z * da, mz * np.abs(z * da)
        if kind == "silu":   # sig (1 + g rest) crosses zero: its two terms
            g = gate_rows(gate, rows, rows_per_gate)
            sig = 1 / (1 + np.exp(-np.clip(g, -700, 700)))
            mg = mz * np.abs(z) * sig * (1 + np.abs(g) * (1 - sig))
        if rows_per_gate == 0:
            out["dgate"], out["dgate_mag"] = dg.sum(0), mg.sum(0)
        else:
            at = np.arange(rows) // rows_per_gate
            out["dgate"], out["dgate_mag"] = np.zeros(gate.shape), np.zeros(gate.shape)
            np.add.at(out["dgate"], at, dg)
            np.add.at(out["dgate_mag"], at, mg)
        dz, mz = dz * a, mz * np.abs(a)
    if gamma_post is not None:
        yh = y * q
        out["dgamma_post"], out["dgamma_post_mag"] = (dz * yh).sum(0), (mz * np.abs(yh)).sum(0)
        v, mv = dz * gamma_post, mz * np.abs(gamma_post)
        dz = q * (v - yh * (v * yh).mean(1, keepdims=True))
        mz = q * (mv + np.abs(yh) * (mv * np.abs(yh)).mean(1, keepdims=True))
    out["dy"], out["dy_mag"] = dz, mz
    return out


def grad_norm(tensors, kind="2"):
    if kind == "2":
        return np.sqrt(sum(float((t * t).sum()) for t in tensors))
    worst = [np.abs(t).max() for t in tensors if t.size]
    return float(np.max(worst)) if worst else 0.0   # (np.max keeps NaN)


def clip_factor(norm, max_norm):
    return min(1.0, max_norm / (norm + 1e-6)) if np.isfinite(norm) else 1.0
