"""The operators at the other end of the model and behind its gradients: embedding lookup with scaling and its
gradient by tokens (alone, or added to the gradient of a head that shares the matrix), layer norm with the
residual sum in front of it (forward, backward), and orthogonalising updates by Newton-Schulz products.

A case is a dict of plain values.  `prepare` makes its inputs on the GPU from the seed alone, `run` is one pass:
the plain form in elementary torch operations, or with `own` set the calls of this library.  `exact` is the same
result in 64 bits.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

IGNORE = -100
EPS = 1e-5          # layer norm
ORTHO_EPS = 1e-7    # added to an update's norm before it divides
STEPS = 5
COEFFICIENTS = (3.4445, -4.7750, 2.0315)
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2}


def _named(name, c):
    return dict(name=name, **c) if name else c


def _embed_case(name, op, tokens, V, H, dtype="bf16", scale=1.0, ignored=0.0, add=False, pad=0):
    """op: embed_fwd, embed_bwd.  ignored: share of tokens that are padding.  add: the gradient is added to
    what the buffer holds (the head's gradient).  pad: elements between the rows of the tokens' matrix."""
    return _named(name, dict(op=op, tokens=tokens, V=V, H=H, dtype=dtype, scale=scale, ignored=ignored, add=add, pad=pad))


def _norm_case(name, op, rows, H, dtype="bf16", residual=True, affine=True, mean=0.5, pad=0):
    """op: ln_fwd, ln_bwd.  residual: x + y is normalised and handed on (backward: its gradient comes back).
    affine: gamma and beta.  mean: of the rows, in standard deviations.  pad: as above, of x or h."""
    return _named(name, dict(op=op, rows=rows, H=H, dtype=dtype, residual=residual, affine=affine, mean=mean, pad=pad))


def _ortho_case(name, count, rows, cols, dtype="bf16", rank=8, spike=1.0, scale=1.0):
    """count updates of rows x cols: noise and, `spike` times as large, a part of low rank."""
    return _named(name, dict(op="ortho", count=count, rows=rows, cols=cols, dtype=dtype, rank=min(rank, rows, cols),
                             spike=spike, scale=scale))


def listed():
    return [
        # one token of a decoding step: latency alone counts
        _embed_case("embed_one_token", "embed_fwd", 1, 128256, 4096),
        # an ordinary large batch, scaled by sqrt(H)
        _embed_case("embed_batch", "embed_fwd", 16384, 152064, 3584, scale=59.87, ignored=0.02),
        # a test-sized model in full precision, tied to its head
        _embed_case("embed_grad_small", "embed_bwd", 256, 4096, 512, "f32", add=True),
        # the tied matrix of a model with a large vocabulary: only the rows of this batch's tokens change
        _embed_case("embed_grad_tied", "embed_bwd", 8192, 256000, 2304, scale=48.0, ignored=0.3, add=True),
        # an embedding of its own: the whole gradient is written, most of its rows are zeros
        _embed_case("embed_grad_whole", "embed_bwd", 16384, 128256, 4096),
        # one token between two blocks
        _norm_case("ln_one_token", "ln_fwd", 1, 4096),
        # the junction of two blocks, the largest batch
        _norm_case("ln_residual", "ln_fwd", 16384, 3584),
        # its backward, an ordinary batch
        _norm_case("ln_grad_residual", "ln_bwd", 8192, 4096),
        # full precision, odd sizes, in front of the first block, rows in a wider buffer
        _norm_case("ln_grad_fp32", "ln_bwd", 2047, 1000, "f32", residual=False, pad=13),
        # a few small projections: launches count
        _ortho_case("ortho_small", 4, 64, 512),
        # the widest matrices of a GPT-2-medium-sized model, one list
        _ortho_case("ortho_model", 24, 4096, 1024, spike=2.0, scale=2.0),
        # full precision, odd sizes
        _ortho_case("ortho_fp32", 2, 1000, 2047, "f32"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def _width(rng, lo, hi):
    """Any residue, half of them multiples of 64."""
    H = _log_uniform(rng, lo, hi)
    return max(lo, H // 64 * 64) if rng.random() < 0.5 else H


def draw(rng):
    """1 .. 32768 tokens of 257 .. 256000 with rows of 64 .. 4096 elements; 1 .. 16384 rows of 64 .. 8192; up to 32
    updates of 16 .. 4096 rows and columns."""
    op = rng.choice(["embed_fwd", "embed_bwd", "embed_bwd", "ln_fwd", "ln_bwd", "ortho", "ortho"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    es = BYTES[dtype]
    pad = rng.choice([0, 0, 0, 8, rng.randint(1, 99)])
    if op.startswith("embed"):
        H = _width(rng, 64, 4096)
        V = _log_uniform(rng, 257, min(256000, 128256 * 8192 // (H * es)))
        tokens = max(1, min(_log_uniform(rng, 1, 32768), 16384 * 8192 // (H * es)))
        return _embed_case("", op, tokens, V, H, dtype, scale=rng.choice([1.0, round(math.sqrt(H), 2)]),
                           ignored=rng.choice([0.0, 0.05, 0.4]), add=op == "embed_bwd" and rng.random() < 0.5, pad=pad)
    if op.startswith("ln"):
        H = _width(rng, 64, 8192)
        rows = max(1, min(_log_uniform(rng, 1, 16384), 16384 * 7168 // (H * es)))
        return _norm_case("", op, rows, H, dtype, residual=rng.random() < 0.6, affine=rng.random() < 0.8,
                          mean=rng.choice([0.0, 0.5, 2.0]), pad=pad)
    short, long = _width(rng, 16, 2048), _width(rng, 64, 4096)
    if short > long:
        short, long = long, short
    most = 24 * 1024 * 1024 * 4096 // (short * short * long * (3 if dtype == "f32" else 1))
    count = max(1, min(_log_uniform(rng, 1, 32), most))
    rows, cols = (short, long) if rng.random() < 0.6 else (long, short)
    return _ortho_case("", count, rows, cols, dtype, rank=rng.randint(1, 16), spike=rng.choice([0.5, 1.0, 2.0]),
                       scale=rng.choice([1.0, 0.2, 2.0]))


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(24101098 + 7919 * int(seed))
    c, dt = case, DTYPES[case["dtype"]]

    def normal(shape, std, mean=0.0, dtype=dt):
        return torch.randn(shape, generator=g, device="cuda").mul_(std).add_(mean).to(dtype)

    s = dict(case=case)
    if c["op"].startswith("embed"):
        # Zipf's law: token k with a probability near 1 / k, as in text under a tokenizer's own order
        u = torch.rand(c["tokens"], generator=g, device="cuda", dtype=torch.float64)
        t = ((c["V"] + 1) ** u).floor().long().clamp_(1, c["V"]) - 1
        t[torch.rand(c["tokens"], generator=g, device="cuda") < c["ignored"]] = IGNORE
        s["tokens"] = t
        if c["op"] == "embed_fwd":
            s["table"] = normal((c["V"], c["H"]), 0.02)
            s["out"] = torch.empty((c["tokens"], c["H"] + c["pad"]), dtype=dt, device="cuda")[:, :c["H"]]
        else:
            s["dout"] = normal((c["tokens"], c["H"] + c["pad"]), 1e-3)[:, :c["H"]]
            s["dtable"] = normal((c["V"], c["H"]), 1e-3) if c["add"] else torch.empty((c["V"], c["H"]), dtype=dt, device="cuda")
        return s
    if c["op"].startswith("ln"):
        rows, H = c["rows"], c["H"]
        length = torch.exp(0.5 * torch.randn(rows, 1, generator=g, device="cuda"))   # rows of different length

        def stream(std, mean=0.0, pad=0):
            wide = torch.randn((rows, H + pad), generator=g, device="cuda").add_(mean).mul_(length * std)
            return wide.to(dt)[:, :H]

        s["gamma"] = normal(H, 0.1, 1.0) if c["affine"] else None
        s["beta"] = normal(H, 0.1) if c["affine"] else None
        if c["op"] == "ln_fwd":
            s["x"] = stream(2.0, c["mean"], c["pad"])
            s["y"] = stream(0.7) if c["residual"] else None
        else:
            s["h"] = stream(2.0, c["mean"], c["pad"])
            s["dn"] = stream(1e-3)
            s["dh"] = stream(1e-3) if c["residual"] else None
        return s
    count, rows, cols, r = c["count"], c["rows"], c["cols"], c["rank"]
    s["updates"] = []
    for _ in range(count):
        left = torch.randn((rows, r), generator=g, device="cuda")
        right = torch.randn((r, cols), generator=g, device="cuda").mul_(c["spike"] / math.sqrt(r))
        s["updates"].append(((left @ right).add_(torch.randn((rows, cols), generator=g, device="cuda"))).mul_(1e-3).to(dt))
    s["outs"] = [torch.empty_like(t) for t in s["updates"]]
    return s


def _in_table(s):
    t, V = s["tokens"], s["case"]["V"]
    return (t != IGNORE) & (t >= 0) & (t < V)


def _plain_embed_fwd(s):
    c = s["case"]
    there = _in_table(s)
    rows = s["table"][torch.where(there, s["tokens"], 0)].float() * c["scale"]
    s["out"].copy_(torch.where(there[:, None], rows, 0.0))
    return s["out"]


def _plain_embed_bwd(s):
    c = s["case"]
    there = _in_table(s)
    at = torch.where(there, s["tokens"], c["V"])          # (one row more for what is left out)
    sums = torch.zeros((c["V"] + 1, c["H"]), device="cuda")
    sums.index_add_(0, at, s["dout"].float())
    sums = sums[:c["V"]].mul_(c["scale"])
    if c["add"]:
        sums.add_(s["dtable"])
    s["dtable"].copy_(sums)
    return s["dtable"]


def _center(h):
    """h - mean and 1 / sqrt(var + eps) of every row."""
    d = h - h.mean(1, keepdim=True)
    return d, 1 / torch.sqrt((d * d).mean(1, keepdim=True) + EPS)


def _plain_ln_fwd(s):
    dt = DTYPES[s["case"]["dtype"]]
    x = s["x"].float()
    z = x if s["y"] is None else x + s["y"].float()
    d, r = _center(z)
    n = d * r
    if s["gamma"] is not None:
        n = n * s["gamma"].float() + s["beta"].float()
    return [None if s["y"] is None else z.to(dt), n.to(dt)]


def _plain_ln_bwd(s):
    dt = DTYPES[s["case"]["dtype"]]
    dn = s["dn"].float()
    d, r = _center(s["h"].float())
    xh = d * r
    u = dn if s["gamma"] is None else dn * s["gamma"].float()
    dx = r * (u - u.mean(1, keepdim=True) - xh * (u * xh).mean(1, keepdim=True))
    if s["dh"] is not None:
        dx = dx + s["dh"].float()
    if s["gamma"] is None:
        return [dx.to(dt), None, None]
    return [dx.to(dt), (dn * xh).sum(0, dtype=torch.float64).to(dt), dn.sum(0, dtype=torch.float64).to(dt)]


def _plain_ortho(s):
    c = s["case"]
    a, b, q = COEFFICIENTS
    X = torch.stack(s["updates"]).float()
    if c["rows"] > c["cols"]:
        X = X.transpose(1, 2).contiguous()
    X = X / ((X.double() ** 2).sum((1, 2), keepdim=True).sqrt() + ORTHO_EPS).float()
    for _ in range(STEPS):
        A = torch.matmul(X, X.transpose(1, 2).contiguous())
        B = b * A + q * torch.matmul(A, A)
        X = a * X + torch.matmul(B, X)
    X = c["scale"] * X
    if c["rows"] > c["cols"]:
        X = X.transpose(1, 2)
    return list(X.to(DTYPES[c["dtype"]]).contiguous().unbind())


def run(s):
    c = s["case"]
    if not own:
        return {"embed_fwd": _plain_embed_fwd, "embed_bwd": _plain_embed_bwd, "ln_fwd": _plain_ln_fwd,
                "ln_bwd": _plain_ln_bwd, "ortho": _plain_ortho}[c["op"]](s)
    import paper_2410_10989_amd as flce
    if c["op"] == "embed_fwd":
        return flce.flce_embedding_fwd(s["table"], s["tokens"], scale=c["scale"], ignore_index=IGNORE, out=s["out"])
    if c["op"] == "embed_bwd":
        return flce.flce_embedding_bwd(s["dout"], s["tokens"], c["V"], scale=c["scale"], ignore_index=IGNORE,
                                       dtable=s["dtable"], accumulate=c["add"])
    if c["op"] == "ln_fwd":
        return list(flce.flce_layer_norm_fwd(s["x"], s["y"], gamma=s["gamma"], beta=s["beta"], eps=EPS))
    if c["op"] == "ln_bwd":
        return list(flce.flce_layer_norm_bwd(s["h"], s["dn"], s["dh"], gamma=s["gamma"], bias=s["beta"] is not None, eps=EPS))
    return flce.flce_orthogonalize(s["updates"], outs=s["outs"], steps=STEPS, coefficients=COEFFICIENTS,
                                   scale=c["scale"], eps=ORTHO_EPS)


def _distinct(c):
    """Distinct tokens to expect among the valid ones."""
    k = np.arange(1, c["V"] + 1, dtype=np.float64)
    p = np.log1p(1 / k) / math.log(c["V"] + 1)
    return float((1 - (1 - p) ** (c["tokens"] * (1 - c["ignored"]))).sum())


def work(case):
    """Every stream read or written once; of a product whose result is symmetric, half."""
    c, es = case, BYTES[case["dtype"]]
    if c["op"] == "embed_fwd":
        return {"bytes": es * c["H"] * (_distinct(c) + c["tokens"]) + 8 * c["tokens"], "flops": c["tokens"] * c["H"]}
    if c["op"] == "embed_bwd":
        valid = c["tokens"] * (1 - c["ignored"])
        written = 2 * _distinct(c) if c["add"] else c["V"]   # (rows that are added to are read, too)
        return {"bytes": es * c["H"] * (valid + written) + 8 * c["tokens"], "flops": valid * c["H"]}
    if c["op"] == "ln_fwd":
        streams, params, per = 2 + 2 * c["residual"], 2 * c["affine"], 5 + c["residual"] + 2 * c["affine"]
        return {"bytes": es * c["H"] * (c["rows"] * streams + params), "flops": per * c["rows"] * c["H"]}
    if c["op"] == "ln_bwd":
        streams, params, per = 3 + c["residual"], 3 * c["affine"], 11 + c["residual"] + 4 * c["affine"]
        return {"bytes": es * c["H"] * (c["rows"] * streams + params), "flops": per * c["rows"] * c["H"]}
    m, n = min(c["rows"], c["cols"]), max(c["rows"], c["cols"])
    return {"bytes": 2 * es * c["count"] * m * n, "flops": c["count"] * STEPS * (3.0 * m * m * n + 1.0 * m * m * m)}


def exact(case, seed):
    s = prepare(case, seed)
    c, wide = case, torch.float64
    if c["op"].startswith("embed"):
        valid = ((s["tokens"] != IGNORE) & (s["tokens"] >= 0) & (s["tokens"] < c["V"])).nonzero()[:, 0]
        tokens = s["tokens"][valid]
        if c["op"] == "embed_fwd":
            out = torch.zeros((c["tokens"], c["H"]), dtype=wide, device="cuda")
            out[valid] = c["scale"] * torch.index_select(s["table"], 0, tokens).to(wide)
            return out
        # runs of equal tokens in sorted order, each added up by itself
        order = torch.sort(tokens, stable=True).indices
        rows, lengths = torch.unique_consecutive(tokens[order], return_counts=True)
        out = s["dtable"].to(wide) if c["add"] else torch.zeros((c["V"], c["H"]), dtype=wide, device="cuda")
        if len(rows):
            sums = torch.segment_reduce(s["dout"][valid[order]].to(wide), "sum", lengths=lengths, axis=0)
            out[rows] += c["scale"] * sums
        return out
    if c["op"].startswith("ln"):
        def normed(h, gamma, beta):
            var, mean = torch.var_mean(h, dim=-1, unbiased=False, keepdim=True)
            n = (h - mean) * (var + EPS).rsqrt()
            return n if gamma is None else torch.addcmul(beta, n, gamma)

        gamma, beta = (None, None) if s["gamma"] is None else (s["gamma"].to(wide).requires_grad_(), s["beta"].to(wide).requires_grad_())
        if c["op"] == "ln_fwd":
            h = s["x"].to(wide) if s["y"] is None else s["x"].to(wide) + s["y"].to(wide)
            return [None if s["y"] is None else h, normed(h, gamma, beta).detach()]
        h = s["h"].to(wide).requires_grad_()
        leaves = [h] if gamma is None else [h, gamma, beta]
        grads = torch.autograd.grad(normed(h, gamma, beta), leaves, s["dn"].to(wide))
        dx = grads[0] if s["dh"] is None else grads[0] + s["dh"].to(wide)
        return [dx, *(grads[1:] or (None, None))]
    # X_k = P_k G with symmetric P_k, a polynomial in G G^T: everything but G itself stays min(rows, cols) wide
    outs = []
    a, b, q = COEFFICIENTS
    for t in s["updates"]:
        G = t.to(wide)
        tall = G.shape[0] > G.shape[1]
        G = G.mT.contiguous() if tall else G
        G = G / (torch.linalg.vector_norm(G) + ORTHO_EPS)
        A = torch.mm(G, G.mT.contiguous())
        P = one = torch.eye(A.shape[0], dtype=wide, device="cuda")
        for _ in range(STEPS):
            f = torch.addmm(a * one, A, torch.addmm(b * one, A, one, alpha=q))   # a + A (b + c A)
            P, A = torch.mm(f, P), torch.linalg.multi_dot([f, A, f])
        X = torch.mm(P, G).mul_(c["scale"])
        outs.append(X.mT if tall else X)
    return outs
