"""The operators in the order in which a training step of a model with a tied embedding uses them: lookup with scaling, a
block's output joined by a layer norm's residual sum, the head on the same matrix, the norm's backward, the gradient of
the lookup added to the head's, all gradients clipped together, the block's matrix update orthogonalised; against
automatic differentiation in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import step_oracle as oracle

pytestmark = pytest.mark.gpu

IGNORE = -100
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def inputs(BT, H, V, dtype):
    g = np.random.Generator(np.random.Philox(key=[BT, H]))
    t = dict(table=0.05 * g.standard_normal((V, H)), M=g.standard_normal((H, H)) / np.sqrt(H),
             gamma=1 + 0.1 * g.standard_normal(H), beta=0.1 * g.standard_normal(H))
    t = {k: torch.from_numpy(v).to(DT[dtype]) for k, v in t.items()}
    tokens = np.floor((V + 1) ** g.random(BT)).astype(np.int64).clip(1, V) - 1
    target = g.integers(0, V, BT)
    tokens[g.random(BT) < 0.1] = IGNORE
    target[g.random(BT) < 0.2] = IGNORE
    return t, torch.from_numpy(tokens), torch.from_numpy(target)


class Step:
    """Buffers of one step and the calls of it."""

    def __init__(self, t, tokens, target, scale, max_norm):
        self.p = {k: v.cuda() for k, v in t.items()}
        self.tokens, self.target, self.scale, self.max_norm = tokens.cuda(), target.cuda(), scale, max_norm

    def run(self):
        import paper_2410_10989_amd as flce
        p = self.p
        V, H = p["table"].shape
        x = flce.flce_embedding_fwd(p["table"], self.tokens, scale=self.scale, ignore_index=IGNORE)
        y = x @ p["M"]
        h, n = flce.flce_layer_norm_fwd(x, y, p["gamma"], p["beta"])
        loss, dn, dtable = flce.flce_fwd_bwd(n, p["table"], self.target, IGNORE)
        dh, dgamma, dbeta = flce.flce_layer_norm_bwd(h, dn, None, p["gamma"])
        dM = x.t() @ dh
        dx = dh + dh @ p["M"].t()
        flce.flce_embedding_bwd(dx, self.tokens, V, scale=self.scale, ignore_index=IGNORE, dtable=dtable, accumulate=True)
        grads = dict(table=dtable, gamma=dgamma, beta=dbeta, M=dM)
        raw = {k: v.clone() for k, v in grads.items()}
        norm = flce.flce_clip_grad_norm(list(grads.values()), self.max_norm)
        update = flce.flce_orthogonalize([dM], outs=[torch.empty_like(dM)])[0]
        return loss, raw, norm, grads, update


def reference(t, tokens, target, scale):
    """Loss and gradients in 64 bits."""
    p = {k: v.double().requires_grad_() for k, v in t.items()}
    x = torch.where((tokens == IGNORE)[:, None], torch.zeros((), dtype=torch.float64), scale * p["table"][tokens.clamp_min(0)])
    h = x + x @ p["M"]
    n = torch.nn.functional.layer_norm(h, h.shape[1:], p["gamma"], p["beta"], 1e-5)
    loss = torch.nn.functional.cross_entropy(n @ p["table"].t(), target, ignore_index=IGNORE)
    loss.backward()
    return loss.item(), {k: v.grad.numpy() for k, v in p.items()}


@pytest.mark.parametrize("BT,H,V,dtype", [(300, 192, 1000, "f32"), (77, 72, 333, "f32"), (300, 192, 1000, "bf16"), (1100, 136, 70, "bf16")])
def test_tied_step(BT, H, V, dtype):
    print(f"case tied step BT={BT} H={H} V={V} {dtype}", flush=True)
    t, tokens, target = inputs(BT, H, V, dtype)
    loss, raw, norm, grads, update = Step(t, tokens, target, 4.0, 0.01).run()
    torch.cuda.synchronize()
    want_loss, want = reference(t, tokens, target, 4.0)
    # fp32: a few hundred terms a sum, 2^-24 each and some factors; bf16 throughout: the bar of the head's own parity tests
    tol = 1e-4 if dtype == "f32" else 2e-2
    assert abs(float(loss) - want_loss) <= (1e-5 if dtype == "f32" else 2e-3) * want_loss
    for k, w in want.items():
        assert np.abs(raw[k].double().cpu().numpy() - w).max() <= tol * np.abs(w).max(), k
    # clipping and the update from exactly these gradients
    ref = {k: v.double().cpu().numpy() for k, v in raw.items()}
    total = np.sqrt(sum((v * v).sum() for v in ref.values()))
    assert total > 0.01 and abs(float(norm) - total) <= 2.0 ** -23 * total
    factor = 0.01 / (total + 1e-6)
    eps = torch.finfo(DT[dtype]).eps / 2
    for k, v in ref.items():
        assert np.all(np.abs(grads[k].double().cpu().numpy() - factor * v) <= (eps + 2.0 ** -22) * np.abs(factor * v) + 2.0 ** -133)
    G = grads["M"].double().cpu().numpy()
    exact, model = oracle.orthogonalize(G), oracle.orthogonalize_rounded(G, 2 if dtype == "f32" else 1)
    off = np.linalg.norm(update.double().cpu().numpy() - exact)
    assert off <= 2 * np.linalg.norm(model - exact) + (eps + 2.0 ** -21) * np.linalg.norm(exact)


def test_captured_step_replays():
    """The whole step in one graph, replayed with other tokens, eager work of another size between the replays."""
    import paper_2410_10989_amd as flce
    t, tokens, target = inputs(400, 128, 500, "bf16")
    s = Step(t, tokens, target, 4.0, 0.01)
    # (the library products of the block are what they are in the graph, too: replays are compared with the eager step)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.run()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = s.run()
    for k in range(4):
        s.tokens.copy_(torch.from_numpy(np.random.Generator(np.random.Philox(key=[k, 9])).integers(0, 500, 400)))
        graph.replay()
        torch.cuda.synchronize()
        got = [out[0].clone(), out[2].clone(), *(v.clone() for v in out[3].values()), out[4].clone()]
        eager = s.run()
        want = [eager[0], eager[2], *eager[3].values(), eager[4]]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        flce.flce_embedding_bwd(torch.randn(5000, 200, device="cuda"), torch.randint(0, 9, (5000,), device="cuda"), 9)
